/*
 * cover.h -- C ABI of the COVER hot path on MI355X (gfx950).
 *
 * COVER (arXiv 2602.06161) verifies previously unmasked "seed" positions inside the same
 * forward pass that drafts new tokens.  This library provides the two per-step device
 * operations of that pass:
 *
 *   cover_attn_fwd      bidirectional attention over the KV-cache-overridden memory with the
 *                       diagonal correction for seed rows (Sec. 5.1; App. B).
 *   cover_select_seeds  stability-aware seed scoring, adaptive budget and top-k
 *                       (Sec. 5.3).
 * and the producers of the selection's inputs:
 *   cover_token_stats   log p of the current token, confidence and argmax per position
 *                       (Sec. 5.3 u(j); Sec. 3 confidence and draft token).
 *   cover_attn_stats    in/out attention masses d_in, d_out over the response region
 *                       (Sec. 5.3 signals).
 * and what a layer needs around them when it decodes one block against a prefix held in an 8-bit
 * cache (Sec. 6.6):
 *   cover_rms_norm      residual addition and root-mean-square norm, also into 8 bits.
 *   cover_rope          rotary positions of queries and keys.
 *   cover_cache_store, cover_cache_load  keys and values into the cache and back.
 *   cover_attn_cached   the block's attention over the cache and its own live rows.
 *
 * Conventions shared by every entry point
 *   - Every data pointer is device memory owned by the caller (hipMalloc, or a framework
 *     allocator).  The library allocates nothing, frees nothing and never synchronises;
 *     work is enqueued on `stream` (0 = the null stream) and runs asynchronously.
 *   - Descriptor and pointer errors are detected on the host before anything is enqueued:
 *     the call then returns COVER_ERR_INVALID or COVER_ERR_UNSUPPORTED and writes nothing.
 *   - COVER_ERR_HIP means the HIP runtime rejected the launch.
 *   - Device-resident arguments (seed lists, seed counts, selection inputs) are not
 *     validated by default; their contract is stated per function.  Violations give
 *     unspecified results but never out-of-bounds memory accesses.  With the environment
 *     variable COVER_DEBUG=1 at the time of a call, the contract is checked on the device
 *     first and violations are recorded (see cover_debug_status).
 *   - Outputs must not alias inputs.
 *   - Where a layer operator's output has strides, its rows must lie apart: in the order of the
 *     strides, each at least the one before times that dimension's size.
 */
#ifndef COVER_H
#define COVER_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  COVER_OK = 0,
  COVER_ERR_INVALID = -1,     /* bad pointer, size, stride or alignment            */
  COVER_ERR_UNSUPPORTED = -2, /* valid request outside what the kernels implement  */
  COVER_ERR_HIP = -3          /* the HIP runtime reported an error at launch       */
} cover_status;

typedef enum { COVER_F32 = 0, COVER_BF16 = 1 } cover_dtype;

/* Largest sequence length the attention kernels accept (the seed bitmap of a sequence is
 * staged in on-chip memory). */
#define COVER_MAX_L 65536
/* Largest selection region per batch row. */
#define COVER_MAX_LR 16384

/*
 * Attention problem description.
 *   B        batch rows (>= 0; 0 is a no-op)
 *   Hq, Hkv  query heads and key/value heads; Hq % Hkv == 0; query head h reads key/value
 *            head h / (Hq / Hkv) (grouped-query attention; Hq == Hkv is plain multi-head)
 *   L        sequence length, prompt plus response (0 is a no-op; <= COVER_MAX_L)
 *   d        head dimension: 64 or 128
 *   max_seeds  row stride of seed_idx (>= 0)
 *   dtype    element type of q, k_live, v_live, k_cache, v_cache and out
 *   scale    score scale; 0 selects 1/sqrt(d) (Sec. 5.1)
 *   q_sb, q_sh, q_sl     element strides of q and out over (batch, head, position)
 *   kv_sb, kv_sh, kv_sl  element strides shared by k_live, v_live, k_cache, v_cache
 * The head dimension is contiguous (stride 1).  Base pointers must be 16-byte aligned and
 * every stride a multiple of 16 bytes' worth of elements.
 */
typedef struct {
  int32_t B, Hq, Hkv, L, d;
  int32_t max_seeds;
  cover_dtype dtype;
  float scale;
  int64_t q_sb, q_sh, q_sl;
  int64_t kv_sb, kv_sh, kv_sl;
} cover_attn_desc;

/*
 * cover_attn_fwd -- COVER attention of one layer (Sec. 5.1 "KV cache override" and
 * "diagonal correction"; App. B.1-B.4).
 *
 * For batch row b with seed set S_b = { seed_idx[b, t] : 0 <= t < n_seed[b] }, query head h
 * and key/value head g:
 *   override memory   K'_j = k_cache[b,g,j] if j in S_b, else k_live[b,g,j]; V' likewise
 *   row view          K^(i) = K', except K^(i)_i = k_live[b,g,i] when i in S_b (the key of
 *                     the masked input); V^(i) likewise
 *   out[b,h,i,:]      = sum_j softmax_j(scale * <q_i, K^(i)_j>) V^(i)_j
 *   lse[b,h,i]        = log sum_j exp(scale * <q_i, K^(i)_j>)   (natural log)
 * Non-seed rows therefore attend to the overridden memory unchanged, and each seed row sees
 * cached states everywhere except its own diagonal, which is the leave-one-out view the
 * paper's closed-form correction (App. B.4) produces.  All scores are kept in fp32 and the
 * softmax is taken over all L positions (non-causal).
 *
 * Arguments
 *   q        [B,Hq,L,d]   queries of the verification input (seeds masked)
 *   k_live, v_live   [B,Hkv,L,d]  keys/values of the verification input
 *   k_cache, v_cache [B,Hkv,L,d]  keys/values cached from the previous step, indexed by
 *                     absolute position; only rows at seed positions are read
 *   seed_idx [B,max_seeds] int32  seed positions; may be NULL when max_seeds == 0
 *   n_seed   [B] int32            seeds per batch row; may be NULL when max_seeds == 0
 *   out      [B,Hq,L,d]   output, same dtype and strides as q
 *   lse      [B,Hq,L] fp32, contiguous; may be NULL
 *   desc     problem description (host memory)
 * Device-data contract: 0 <= n_seed[b] <= max_seeds; seed_idx[b,0..n_seed[b]) distinct and in
 * [0, L) (any order).  n_seed outside [0, max_seeds] is clamped into it and entries outside
 * [0, L) are ignored.
 * Returns COVER_ERR_UNSUPPORTED for d not in {64, 128} or L > COVER_MAX_L.
 */
cover_status cover_attn_fwd(const void* q, const void* k_live, const void* v_live,
                            const void* k_cache, const void* v_cache,
                            const int32_t* seed_idx, const int32_t* n_seed,
                            void* out, float* lse,
                            const cover_attn_desc* desc, hipStream_t stream);

/*
 * Selection description.
 *   B           batch rows (>= 0)
 *   Lr          candidate region length per row (>= 0, <= COVER_MAX_LR)
 *   max_seeds   row stride / capacity of seed_idx (>= 0)
 *   pos_offset  added to every emitted position (the region's start in the sequence)
 */
typedef struct {
  int32_t B, Lr;
  int32_t max_seeds;
  int32_t pos_offset;
} cover_select_desc;

/*
 * cover_select_seeds -- stability-aware seed selection with an adaptive revision rate
 * (Sec. 5.3 "Stability aware seed scoring", "Adaptive revision rate").
 *
 * Per batch row, over region positions j in [0, Lr):
 *   flags bit 0 = j is unmasked (j in U_t); bit 1 = j is excluded (a seed of the previous
 *   step, or its ReMask budget is used up); other bits are ignored.
 *   score s_j   = ((-(double)logp_j) * (1 + (double)d_in_j)) / (1 + (double)d_out_j), for j
 *                 in U_t, in IEEE fp64 with round-to-nearest and this exact association
 *   mean        = (sum of s_j over U_t) / |U_t|, the sum taken as a stride-halving tree over
 *                 the region zero-padded to the next power of two
 *   budget      = least k >= 0 with k*k >= c, c = #{ j in U_t : s_j > mean } (= n_t pi_t)
 *   selection   = the min(budget, #eligible, max_seeds) eligible positions (in U_t, not
 *                 excluded) ranked first by score descending then position ascending
 * Outputs
 *   seed_idx [B,max_seeds] int32: selected positions + pos_offset in ascending order,
 *            then -1; n_seed [B] int32: how many; score [B,Lr] fp64 (may be NULL): s_j on
 *            U_t, 0 elsewhere.  The results are bit-exact functions of the inputs.
 * Inputs: logp, d_in, d_out fp32 [B,Lr] row-major (logp = log p_j(y_j) <= 0, the model's
 * log-probability of the token currently at j; d_in, d_out >= 0 are the in/out attention
 * masses); flags uint8 [B,Lr].  Values at positions outside U_t are ignored (they may be
 * anything, including non-finite).  Device-data contract: values on U_t finite, d_in and
 * d_out >= 0.
 * The output layout matches cover_attn_fwd's seed_idx / n_seed, so the next step's
 * attention can consume it without a host round-trip.
 */
cover_status cover_select_seeds(const float* logp, const float* d_in, const float* d_out,
                                const uint8_t* flags,
                                int32_t* seed_idx, int32_t* n_seed, double* score,
                                const cover_select_desc* desc, hipStream_t stream);

/*
 * Token statistics description.
 *   R           rows (positions; >= 0, 0 is a no-op)
 *   V           vocabulary size (>= 1)
 *   dtype       element type of logits (COVER_BF16 or COVER_F32)
 *   row_stride  elements between consecutive rows of logits (>= V); the base pointer and
 *               row_stride * element size must be multiples of 16 bytes
 */
typedef struct {
  int32_t R, V;
  cover_dtype dtype;
  int64_t row_stride;
} cover_token_desc;

/*
 * cover_token_stats -- per-position statistics of the model's output distribution
 * (Sec. 5.3: u(j) = -log p_j(y_j); Sec. 3: confidence = max_v p_j(v), draft token = argmax).
 *
 * For row r with logits x_r[0..V) and lz_r = log sum_v exp(x_r[v]) (natural log):
 *   logp[r]   = x_r[tokens[r]] - lz_r
 *   conf[r]   = exp(max_v x_r[v] - lz_r)
 *   argmax[r] = the smallest v attaining max_v x_r[v]
 * Arithmetic in fp32 (exp/log of the exp2/log2 units); one pass over the logits (a second over
 * rows whose maximum is beyond 1e30 in size).
 * Arguments: logits [R, row_stride] (device); tokens int32 [R] (device; may be NULL when
 * logp is NULL); logp, conf fp32 [R] and argmax int32 [R] (device outputs, each may be
 * NULL).  Device-data contract: tokens in [0, V) (a token outside gives logp = NaN, never
 * an out-of-bounds read); logits finite or -inf (a masked token).  argmax is in [0, V) whatever
 * the row holds.
 */
cover_status cover_token_stats(const void* logits, const int32_t* tokens,
                               float* logp, float* conf, int32_t* argmax,
                               const cover_token_desc* desc, hipStream_t stream);

/*
 * cover_token_sample -- temperature sampling of the draft tokens (the stochastic decoding of
 * the paper's appendix on robustness): per row r of logits (same description and layout
 * rules as cover_token_stats),
 *   token[r] = argmax_v (x_v / T + g_v), g_v = -ln(-ln u_v) (Gumbel-max: a draw from
 *              softmax(x / T); the smallest v on ties)
 *   prob[r]  = softmax(x / T) at token[r] (the confidence compared with the drafting
 *              threshold; may be NULL)
 * u_v = ((w >> 9) + 1/2) 2^-23 with w word v % 4 of Philox4x32-10 (Salmon et al., SC 2011)
 * at counter (v / 4, r, step, 0) and key (seed mod 2^32, seed >> 32): a fixed function of
 * (seed, step, row, token), reproducible across launches and devices.  x_v / T + g_v is
 * compared in fp64 (with g_v from fp32 logarithms), softmax(x / T) summed in fp32.  temperature:
 * > 0 and finite.  Logits finite or -inf; token is in [0, V) whatever the row holds.  token int32
 * [R], prob fp32 [R]: device outputs.
 */
cover_status cover_token_sample(const void* logits, float temperature, uint64_t seed, uint32_t step,
                                int32_t* token, float* prob, const cover_token_desc* desc,
                                hipStream_t stream);

/*
 * Attention-mass description: the attention problem of cover_attn_fwd (same fields and
 * stride rules; bf16 only) plus the response region [r0, r0 + Lr).
 *   r0, Lr      0 <= r0, 1 <= Lr, r0 + Lr <= L (Lr == 0 is a no-op)
 */
typedef struct {
  cover_attn_desc attn;
  int32_t r0, Lr;
} cover_stats_desc;

/* Largest response region cover_attn_stats accepts. */
#define COVER_STATS_MAX_LR 2048
/* An upper bound of the workspace of cover_attn_stats in floats, valid for every launch:
 * B * Hq * (1 + ceil(Lr / 32)) * Lr.  cover_attn_stats_workspace gives what a call asks for. */
#define COVER_ATTN_STATS_WORKSPACE(B, Hq, Lr) \
  ((int64_t)(B) * (Hq) * (1 + ((int64_t)(Lr) + 31) / 32) * (Lr))

/*
 * cover_attn_stats -- the in/out attention masses of Sec. 5.3 from the last layer's
 * corrected attention weights, averaged over query heads, restricted to the response region.
 *
 * With w^(h)_{i,j} = exp(scale <q_i, K^(i)_j> - lse[b,h,i]) the weights of cover_attn_fwd
 * (override memory, leave-one-out view for seed rows, normalised over all L positions by
 * the lse that call returned) and A_{i->j} = (1/Hq) sum_h w^(h)_{i,j}, for region positions
 * j = r0 + t, t in [0, Lr):
 *   d_in[b,t]  = sum over region rows i with masked[b, i-r0]  of A_{i->j}
 *   d_out[b,t] = sum over region columns i with drafted[b, i-r0] of A_{j->i}
 * Arguments: q, k_live, k_cache, seed_idx, n_seed as for cover_attn_fwd (v is not needed);
 * lse fp32 [B,Hq,L] contiguous, as returned by cover_attn_fwd for the same inputs;
 * masked, drafted uint8 [B,Lr] (nonzero = member; device); d_in, d_out fp32 [B,Lr]
 * (device outputs); workspace: device fp32 buffer of at least
 * cover_attn_stats_workspace(B, Hq, Lr) floats (COVER_ATTN_STATS_WORKSPACE(B, Hq, Lr) always
 * suffices) owned by the caller (its contents on entry are ignored, on exit unspecified).
 * Two kernel launches on `stream`; partial sums are added in a fixed order, so the results
 * are deterministic.  Weights are formed in fp32 from the fp32 lse.
 * Returns COVER_ERR_UNSUPPORTED for a dtype other than bf16, d not in {64, 128},
 * L > COVER_MAX_L or Lr > COVER_STATS_MAX_LR.
 */
cover_status cover_attn_stats(const void* q, const void* k_live, const void* k_cache,
                              const int32_t* seed_idx, const int32_t* n_seed, const float* lse,
                              const uint8_t* masked, const uint8_t* drafted,
                              float* d_in, float* d_out, float* workspace,
                              const cover_stats_desc* desc, hipStream_t stream);

/*
 * cover_attn_stats_workspace -- floats of workspace a cover_attn_stats call with these B, Hq
 * and Lr asks for: B * Hq * (1 + G) * Lr, with G the number of workgroups per head that the
 * launch divides the region's 32-position tiles among (about 256 workgroups in all; G <=
 * ceil(Lr / 32)).  The kernels use at most that, now two rows of Lr floats per head.  A host
 * function: no GPU work.  Returns -1 for negative arguments.
 */
int64_t cover_attn_stats_workspace(int32_t B, int32_t Hq, int32_t Lr);

/* Floats of the library's own per-GPU workspace behind cover_attn_stats_noalloc (4 MiB). */
#define COVER_STATS_SCRATCH_FLOATS (1 << 20)

/*
 * cover_attn_stats_noalloc -- cover_attn_stats without a workspace argument, for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving loops, hosts
 * that forbid allocation).  Same arguments, results and checks as cover_attn_stats, except
 * that the partial sums go to a fixed array inside the library: COVER_STATS_SCRATCH_FLOATS
 * floats on each GPU the library runs on, held until the process ends (its device address is
 * looked up on the first call on each GPU; nothing is allocated, by this call or any other).
 * Every call on one GPU shares that array and the work it enqueues reads back only what the
 * same call wrote, so calls that run one after another (on one stream, or ordered by events)
 * are independent; calls that can overlap on one GPU (different streams with no ordering)
 * race on the array and give unspecified results.
 * Returns COVER_ERR_UNSUPPORTED when cover_attn_stats_workspace(B, Hq, Lr) exceeds
 * COVER_STATS_SCRATCH_FLOATS (for instance B * Hq > 256 at Lr = 2048, or B * Hq > 1024 at
 * Lr = 512), before anything is enqueued; COVER_ERR_HIP if the array's address cannot be
 * obtained.
 */
cover_status cover_attn_stats_noalloc(const void* q, const void* k_live, const void* k_cache,
                                      const int32_t* seed_idx, const int32_t* n_seed,
                                      const float* lse, const uint8_t* masked,
                                      const uint8_t* drafted, float* d_in, float* d_out,
                                      const cover_stats_desc* desc, hipStream_t stream);

/*
 * Block-query attention description: the attention problem of cover_attn_fwd (same fields
 * and stride rules, with attn.L the number of keys; q and out hold Lq rows at the q strides)
 * plus the query block [q_off, q_off + Lq) and the number of key splits.
 *   q_off, Lq   0 <= q_off, 0 <= Lq, q_off + Lq <= attn.L (Lq == 0 is a no-op)
 *   n_split     1 <= n_split <= 256.  1: one launch, one workgroup per 32 query rows whose
 *               waves split the keys among themselves (no workspace).  > 1: the keys are cut
 *               into at most n_split ranges (fewer where those finish sooner, one included)
 *               processed by separate workgroups and merged by a second launch (more
 *               workgroups per query row; the partial results go through the workspace)
 */
typedef struct {
  cover_attn_desc attn;
  int32_t q_off, Lq;
  int32_t n_split;
} cover_rect_desc;

/* 4-byte words per (row, split) record of the cover_attn_rect workspace. */
#define COVER_RECT_RECORD 68
/* Workspace of cover_attn_rect in floats (none for n_split == 1). */
#define COVER_ATTN_RECT_WORKSPACE(B, Hq, Lq, n_split) \
  ((n_split) > 1 ? (int64_t)(B) * (Hq) * (n_split) * (Lq) * COVER_RECT_RECORD : (int64_t)0)

/*
 * cover_attn_rect -- COVER attention for one block of query rows against all L keys (the
 * prefix-cache decoding COVER is combined with in Sec. 6.6: the block's rows are recomputed,
 * the other positions' keys and values are reused).
 *
 * Row r of out/lse is row q_off + r of what cover_attn_fwd computes for a length-L sequence
 * with the same k_live, v_live, k_cache, v_cache and seeds (Sec. 5.1 override memory and
 * the leave-one-out diagonal of a seed row, App. B): q holds only the block's Lq rows.
 * Seeds may lie anywhere in [0, L), inside the block or not.
 * Arguments as for cover_attn_fwd; out [B,Hq,Lq,d] at the q strides; lse fp32 [B,Hq,Lq]
 * contiguous (may be NULL); workspace: for n_split > 1 a device fp32 buffer of
 * COVER_ATTN_RECT_WORKSPACE(B, Hq, Lq, n_split) floats owned by the caller (contents on
 * entry ignored, on exit unspecified); for n_split == 1 not used (may be NULL).  One kernel
 * launch on `stream` for one range of the keys, two otherwise (partial results per range, then
 * a merge; past 2^23 workgroups the first in several); every sum runs in a fixed order, so
 * results are deterministic.
 * Returns COVER_ERR_UNSUPPORTED for a dtype other than bf16, d != 128, L > COVER_MAX_L, or
 * n_split == 1 with kv_sl >= 2^26.
 */
cover_status cover_attn_rect(const void* q, const void* k_live, const void* v_live,
                             const void* k_cache, const void* v_cache,
                             const int32_t* seed_idx, const int32_t* n_seed,
                             void* out, float* lse, float* workspace,
                             const cover_rect_desc* desc, hipStream_t stream);

/*
 * Decoding-state update description.
 *   B              batch rows (>= 0; 0 is a no-op)
 *   Lr             region length per row (>= 0, <= COVER_MAX_LR)
 *   max_seeds      row stride / capacity of seed_idx (>= 0)
 *   pos_offset     absolute position of region index 0 (seed_idx holds absolute positions)
 *   mask_id        the [MASK] token id
 *   draft_cap      most positions drafted per row and step (>= 0)
 *   remask_budget  ReMasks after which a position is no longer selectable as a seed
 *   tau            confidence threshold (not NaN), used for drafting and for Replace
 *   min_draft      0 <= min_draft <= draft_cap; 0 is the paper's rule.  Otherwise, when fewer
 *                  than min_draft masked positions pass tau, the min_draft most confident
 *                  masked positions (same order; NaN confidences never drafted) are drafted
 *                  instead, so a decoding loop always progresses (not in the paper)
 */
typedef struct {
  int32_t B, Lr;
  int32_t max_seeds;
  int32_t pos_offset;
  int32_t mask_id;
  int32_t draft_cap;
  int32_t remask_budget;
  float tau;
  int32_t min_draft;
} cover_update_desc;

/*
 * cover_decode_update -- one step's update of the decoding state (Sec. 5.2 drafting and
 * revision outcomes, Sec. 3 state update, Sec. 5.3 ReMask budget and exclusion), per row:
 *   drafting   D = the masked positions (tokens == mask_id) with conf > tau, compared in
 *              fp32; if more than draft_cap qualify, the draft_cap largest by (conf
 *              descending, position ascending).  Each takes its argmax token.
 *   revision   each previous seed i (seed_idx[b, :n_seed[b]] - pos_offset; entries outside
 *              [0, Lr) or at masked positions are ignored, repeats count once):
 *              Keep if argmax_i == tokens_i; else Replace (tokens_i = argmax_i) if
 *              conf_i > tau; else ReMask (tokens_i = mask_id, remask_count_i += 1).
 *   flags      bit 0 = unmasked after the update; bit 1 = i was a seed, or
 *              remask_count_i >= remask_budget -- the flags cover_select_seeds takes next.
 * Arguments (all device memory, row-major [B,Lr] unless stated):
 *   tokens int32 (in/out; the state U/M of the region), argmax int32 and conf fp32 (the
 *   step's argmax token and its probability, e.g. from cover_token_stats), seed_idx int32
 *   [B,max_seeds] and n_seed int32 [B] (the seeds of the step, as cover_select_seeds
 *   emits them; may be NULL when max_seeds == 0), remask_count int32 (in/out),
 *   flags uint8 (out, may be NULL), drafted uint8 (out, 1 = drafted this step, may be NULL),
 *   counts int32 [B,5] (out, may be NULL): |D|, kept, replaced, remasked, masked after;
 *   last_unmask int32 (in/out, may be NULL): the token of each position's most recent
 *   [MASK] -> token transition (-1 = none yet); every drafted position records its new
 *   token (Replace is not an unmasking and leaves it alone);
 *   flipflops int32 [B] (out, may be NULL; needs last_unmask): flip-flop events of the
 *   step (Sec. 4 definition): drafted positions whose new token equals their last_unmask
 *   entry on entry.
 * One kernel launch on `stream`; every result is an exact function of the inputs.  n_seed
 * values outside [0, max_seeds] are clamped.
 */
cover_status cover_decode_update(int32_t* tokens, const int32_t* argmax, const float* conf,
                                 const int32_t* seed_idx, const int32_t* n_seed,
                                 int32_t* remask_count, uint8_t* flags, uint8_t* drafted,
                                 int32_t* counts, int32_t* last_unmask, int32_t* flipflops,
                                 const cover_update_desc* desc, hipStream_t stream);

/*
 * The operators of a layer that decodes one block against a prefix held in an 8-bit cache (the
 * prefix-cache decoding of Sec. 6.6): the norm before a projection, rotary positions of its
 * queries and keys, the cache written and read back, and the attention that reads it.
 *
 * The e4m3 form of a row x of numbers (OCP 8-bit floats of 4 exponent and 3 mantissa bits):
 *   scale = max(max_i |x_i| / 448, 2^-126), fp32;  code_i = x_i * (1 / scale) in fp32, rounded to
 *   the nearest e4m3, ties to even.  The row stands for scale * code_i: off by at most 2^-4 of
 *   x_i, or 2^-10 scale where that is more.  A row of zeros has scale 2^-126; a row that holds an
 *   infinity or a NaN stands for NaN throughout.
 */

/*
 * Norm description.
 *   R, D        rows (>= 0; 0 is a no-op) and elements per row (1 <= D <= COVER_NORM_MAX_D)
 *   dtype       element type of x, residual, weight, residual_out, and of out without scale
 *   eps         added to the mean square; >= 0, finite
 *   *_stride    elements between consecutive rows (>= D; not read where R is 1, res_stride and
 *               res_out_stride not where their tensor is NULL).  Base pointers and strides in bytes are
 *               multiples of 16 (for out in e4m3 too).
 */
typedef struct {
  int32_t R, D;
  cover_dtype dtype;
  float eps;
  int64_t x_stride, res_stride, res_out_stride, out_stride;
} cover_norm_desc;

/* Longest row cover_rms_norm accepts. */
#define COVER_NORM_MAX_D 32768

/*
 * cover_rms_norm -- the residual's addition and the root-mean-square norm, per row r:
 *   h          = x + residual in fp32 (x alone without a residual)
 *   residual_out[r] = h rounded to dtype (not written where NULL)
 *   y          = (h * (1 / sqrt(mean_i h_i^2 + eps))) * weight in fp32, from the unrounded h
 *   out[r]     = y rounded to dtype; with scale != NULL y's e4m3 form: out holds the codes, one byte
 *               each, and scale[r] the row's scale
 * Arguments: x [R, x_stride]; residual [R, res_stride] or NULL; weight [D] contiguous or NULL
 * (ones); residual_out or NULL; out [R, out_stride]; scale fp32 [R] or NULL.  residual_out may be x
 * or residual, and out (without scale) may be x, where the strides are the same.  Sums in fp32 in a
 * fixed order: results are deterministic.  Squares beyond fp32 (|h| above 1e19) give zeros or NaN; those
 * that vanish there (below 1e-22) count as 0 beside eps.
 * One kernel launch.  Returns COVER_ERR_UNSUPPORTED for D > COVER_NORM_MAX_D and for rows of more than 2^32 - 1
 * threads together (at most 1024 per row; fewer than 2^22 rows always fit).
 */
cover_status cover_rms_norm(const void* x, const void* residual, const void* weight,
                            void* residual_out, void* out, float* scale,
                            const cover_norm_desc* desc, hipStream_t stream);

/* How cover_rope_freq scales frequencies for contexts longer than the model was trained on. */
typedef enum {
  COVER_ROPE_PLAIN = 0,   /* f_i = base^(-2 i / rot) / (2 pi) turns per position                   */
  COVER_ROPE_LINEAR = 1,  /* f_i / factor: positions interpolated                                  */
  COVER_ROPE_BASE = 2,    /* base * factor^(rot / (rot - 2)) in base's place: the slowest frequency
                             interpolated, the fastest kept                                        */
  COVER_ROPE_PARTS = 3    /* with t = original_length * f_i turns over the original context and
                             g = clamp((t - low) / (high - low), 0, 1): f_i (g + (1 - g) / factor) */
} cover_rope_scaling;

/*
 * cover_rope_freq -- the table of rot / 2 frequencies, in turns per position, that cover_rope
 * takes (Su et al. 2021; interpolation: Chen et al. 2023; by parts: Peng et al. 2023).  A host
 * function: freq is host memory, the caller copies it to the GPU once.  rot even and >= 2 (>= 4
 * for COVER_ROPE_BASE); base > 1; factor >= 1; original_length >= 1 and low < high for
 * COVER_ROPE_PARTS (not read otherwise).
 */
cover_status cover_rope_freq(double* freq, int32_t rot, double base, cover_rope_scaling scaling,
                             double factor, double original_length, double low, double high);

/*
 * Rotary description.
 *   B, L        batch rows and positions per row (>= 0; 0 is a no-op)
 *   Hq, Hkv     heads of q and of k (>= 0)
 *   d, rot      head dimension (64 or 128); rotated elements at its front: even, 0 < rot <= d
 *   interleaved 0: elements i and i + rot / 2 form pair i; 1: elements 2 i and 2 i + 1
 *   dtype       element type of all four tensors
 *   attention_factor  factor on the rotated elements (finite; 1 without frequency scaling)
 *   pos_sb      elements between the batch rows of pos (0: one row for all)
 *   *_sb, *_sh, *_sl  element strides over (batch, head, position); the head dimension is
 *               contiguous, base pointers and strides multiples of 16 bytes
 */
typedef struct {
  int32_t B, L, Hq, Hkv, d, rot, interleaved;
  cover_dtype dtype;
  float attention_factor;
  int64_t pos_sb;
  int64_t q_sb, q_sh, q_sl, qo_sb, qo_sh, qo_sl;
  int64_t k_sb, k_sh, k_sl, ko_sb, ko_sh, ko_sl;
} cover_rope_desc;

/*
 * cover_rope -- rotary positions of queries and keys: with a = 2 pi pos[b, l] freq[i], the pair
 * (x, y) number i of every head becomes attention_factor * (x cos a - y sin a, y cos a + x sin a);
 * elements from rot on are copied.  The angle's turns are reduced in fp64, so far positions lose
 * nothing; sine, cosine and the rotation are in fp32, rounded once to dtype.
 * Arguments: q [B,Hq,L,d], k [B,Hkv,L,d]; pos int32 [B,L] (any value, also negative); freq fp64
 * [rot / 2], in turns per position; q_out, k_out.  k and k_out may be NULL where Hkv == 0, q and
 * q_out where Hq == 0.  q_out may be q and k_out may be k with the same strides; any other two of the
 * four at one address are refused where one of them is an output.  One kernel launch.
 */
cover_status cover_rope(const void* q, const void* k, const int32_t* pos, const double* freq,
                        void* q_out, void* k_out, const cover_rope_desc* desc, hipStream_t stream);

/*
 * Description of the 8-bit cache's rows that a call writes or reads.
 *   B, H        batch rows, key/value heads (>= 0)
 *   N           rows per batch row of the call (>= 0; any of B, H, N 0 is a no-op)
 *   L           positions the cache holds (>= 1)
 *   d           head dimension (64 or 128)
 *   first       position of row 0 where pos is NULL (rows first, first + 1, ...)
 *   dtype       element type of k and v
 *   k_sb .. v_sl  element strides of k and v over (batch, head, row); head dimension contiguous,
 *               base pointers and strides multiples of 16 bytes
 *   c_sb, c_sh, c_sl  strides in bytes shared by the code tensors; multiples of 16
 *   s_sb, s_sh  strides in floats shared by the scale tensors (positions are contiguous)
 */
typedef struct {
  int32_t B, H, N, L, d, first;
  cover_dtype dtype;
  int64_t k_sb, k_sh, k_sl, v_sb, v_sh, v_sl;
  int64_t c_sb, c_sh, c_sl;
  int64_t s_sb, s_sh;
} cover_cache_desc;

/*
 * cover_cache_store -- keys and values written into the 8-bit cache: row n of batch row b and head
 * h of k goes to position p = pos[b, n] (or first + n) of k_codes and k_scale in e4m3 form (one
 * scale per head and position), v likewise.  Rows whose position is outside [0, L) are skipped, and
 * positions that no row names keep what they held.
 * Arguments: k, v [B,H,N,d]; pos int32 [B,N] contiguous or NULL; k_codes, v_codes e4m3 [B,H,L,d];
 * k_scale, v_scale fp32 [B,H,L].  Device-data contract: the positions in [0, L) of a batch row are
 * distinct (a position listed twice holds codes and a scale of either row).  One kernel launch.
 */
cover_status cover_cache_store(const void* k, const void* v, const int32_t* pos,
                               void* k_codes, void* v_codes, float* k_scale, float* v_scale,
                               const cover_cache_desc* desc, hipStream_t stream);

/*
 * cover_cache_load -- rows of the 8-bit cache read back: row n of k is scale * code of position
 * pos[b, n] (or first + n) in fp32, rounded to dtype; v likewise.  Rows whose position is outside
 * [0, L) are zeros.  Positions may repeat.  Arguments as for cover_cache_store, k and v written.
 */
cover_status cover_cache_load(void* k, void* v, const int32_t* pos, const void* k_codes,
                              const void* v_codes, const float* k_scale, const float* v_scale,
                              const cover_cache_desc* desc, hipStream_t stream);

/* Longest block of query rows cover_attn_cached accepts. */
#define COVER_CACHED_MAX_LQ 2048

/*
 * Description of block attention over the 8-bit cache.
 *   B, Hq, Hkv  batch rows (>= 0; 0 is a no-op), query heads, key/value heads (Hq % Hkv == 0)
 *   L           positions the cache holds, the most keys a row can have (<= COVER_MAX_L)
 *   Lq          query rows per batch row (>= 0; 0 is a no-op; <= COVER_CACHED_MAX_LQ)
 *   d           head dimension: 64 or 128
 *   max_seeds   row stride of seed_idx (>= 0)
 *   q_off       position of query row 0 where off is NULL: 0 <= q_off, q_off + Lq <= L
 *   n_split     1 <= n_split <= 256: the keys are cut into at most n_split ranges (fewer where those
 *               finish sooner) whose partial results go through the workspace and are joined by a
 *               second launch; 1: one launch
 *   scale       score scale; 0 selects 1/sqrt(d)
 *   q_sb, q_sh, q_sl, o_...     element strides of q and of out over (batch, head, row)
 *   k_sb, k_sh, k_sl, v_...     element strides of k_live and of v_live
 *   c_sb, c_sh, c_sl, s_sb, s_sh  strides of the cache, as in cover_cache_desc
 */
typedef struct {
  int32_t B, Hq, Hkv, L, Lq, d, max_seeds, q_off, n_split;
  float scale;
  int64_t q_sb, q_sh, q_sl, o_sb, o_sh, o_sl;
  int64_t k_sb, k_sh, k_sl, v_sb, v_sh, v_sl;
  int64_t c_sb, c_sh, c_sl;
  int64_t s_sb, s_sh;
} cover_cached_desc;

/*
 * cover_attn_cached_splits -- the n_split that suits a cover_attn_cached call of these sizes (1 where
 * the workgroups of one launch fill the GPU or the keys are few).  A host function: no GPU work.
 * Returns 1 for sizes that cover_attn_cached rejects.
 */
int32_t cover_attn_cached_splits(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int32_t Lq);

/*
 * cover_attn_cached_plan -- how a cover_attn_cached call of these sizes runs: *ranges, the key ranges it
 * takes (at most n_split), and *rows, the query rows per workgroup (32, 64 or 128).  A host function.
 * Sizes and n_split that cover_attn_cached rejects, and empty ones, are rejected here too.
 */
cover_status cover_attn_cached_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int32_t Lq, int32_t d,
                                    int32_t n_split, int32_t* ranges, int32_t* rows);

/* Workspace of cover_attn_cached in floats (none for n_split == 1). */
#define COVER_ATTN_CACHED_WORKSPACE(B, Hq, Lq, d, n_split) \
  ((n_split) > 1 ? (int64_t)(B) * (Hq) * (n_split) * (Lq) * ((d) + 4) : (int64_t)0)

/*
 * cover_attn_cached -- COVER attention for one block of query rows whose other positions' keys and
 * values are held in the 8-bit cache (Sec. 5.1 and App. B for each row; Sec. 6.6).
 *
 * Batch row b has len = kv_len[b] keys (L where kv_len is NULL) and its block starts at
 * o = off[b] (q_off where off is NULL); query row r is position o + r and exists where
 * o + r < len.  With S_b the seeds as for cover_attn_fwd, for positions j < len:
 *   memory     K'_j = k_live row j - o if j lies in the block and not in S_b, else the cache's
 *              position j (scale * code); V' likewise
 *   row view   a seed row sees its own live key and value on its diagonal, as in cover_attn_fwd
 *   out, lse   as for cover_attn_fwd, over the keys [0, len)
 * Rows that do not exist (o + r >= len) are not written, neither in out nor in lse; positions at or
 * past len are not read.  Seeds outside the block change nothing.
 * Arguments: q, out [B,Hq,Lq,d] bf16; k_live, v_live [B,Hkv,Lq,d] bf16, the block's rows; k_codes,
 * v_codes e4m3 [B,Hkv,L,d] and k_scale, v_scale fp32 [B,Hkv,L] as cover_cache_store writes them;
 * off, kv_len int32 [B] or NULL; seed_idx, n_seed as for cover_attn_fwd (absolute positions); lse fp32
 * [B,Hq,Lq] contiguous or NULL; workspace: for n_split > 1 a device buffer of
 * COVER_ATTN_CACHED_WORKSPACE(B, Hq, Lq, d, n_split) floats, 16-byte aligned (contents on entry
 * ignored, on exit unspecified).  Scores, softmax and sums in fp32, in a fixed order: results are
 * deterministic.  A cached key's weight times its value's scale is rounded to fp16: off by at most 2^-11
 * of itself, or by 2^-28 of the row's largest weight times the largest value scale read (or times 2^-30,
 * where all are less); live rows' weights to 2^-16, or 2^-126 of that product.  Weights of up to 2^9 times
 * values are summed in fp32 before they are divided: values beyond 2^76 may give infinities.  Scores up to
 * fp32's largest number are taken as they are rounded, where scale times a key's scale is such a number too.
 * Device-data contract: as for seeds; 0 <= off[b] <= kv_len[b] <= L (values outside are clamped: kv_len into
 * [0, L], off into [0, kv_len]).
 * Returns COVER_ERR_UNSUPPORTED for d not in {64, 128}, L > COVER_MAX_L, Lq > COVER_CACHED_MAX_LQ or
 * more than 2^23 - 8 workgroups (one per 32 rows of the query heads of a key/value head, and range) or
 * 2^24 - 4 rows (B * Hq * Lq).
 */
cover_status cover_attn_cached(const void* q, const void* k_live, const void* v_live,
                               const void* k_codes, const void* v_codes,
                               const float* k_scale, const float* v_scale,
                               const int32_t* off, const int32_t* kv_len,
                               const int32_t* seed_idx, const int32_t* n_seed,
                               void* out, float* lse, float* workspace,
                               const cover_cached_desc* desc, hipStream_t stream);

/*
 * cover_debug_status -- the contract checks enabled by COVER_DEBUG=1 (a debugging aid for
 * integrations; not for production paths).
 *
 * While the environment variable COVER_DEBUG is "1", every cover_attn_fwd, cover_attn_rect,
 * cover_attn_cached and cover_attn_stats call first checks its seed lists, every
 * cover_select_seeds call its inputs on U_t, and every cover_cache_store call its list of
 * positions (in [0, COVER_MAX_L)), with a small kernel on the same stream; a violation sets bits of
 * a status word kept on the current GPU:
 */
#define COVER_DEBUG_SEED_COUNT 1        /* some n_seed[b] outside [0, max_seeds]            */
#define COVER_DEBUG_SEED_RANGE 2        /* a listed seed position outside [0, L)             */
#define COVER_DEBUG_SEED_DUPLICATE 4    /* a seed position listed twice in one batch row     */
#define COVER_DEBUG_SELECT_NONFINITE 8  /* logp, d_in or d_out not finite at a j in U_t      */
#define COVER_DEBUG_SELECT_NEGATIVE 16  /* d_in or d_out negative at a j in U_t              */
#define COVER_DEBUG_STORE_DUPLICATE 32  /* a cache position stored twice in one batch row    */
/*
 * cover_debug_status copies that word of the current GPU to *status (host memory) after
 * the work already enqueued on `stream` and, if clear != 0, resets it to 0.  Unlike every
 * other entry point it waits for `stream` to finish before returning.  Bits accumulate
 * across calls until cleared; the word starts at 0.  Returns COVER_ERR_INVALID for a NULL
 * status, COVER_ERR_HIP if the copy fails.
 */
cover_status cover_debug_status(int32_t* status, int32_t clear, hipStream_t stream);

/* Static string naming a status code. */
const char* cover_status_str(cover_status s);

/* Library version as major*10000 + minor*100 + patch. */
int32_t cover_version(void);

#ifdef __cplusplus
}
#endif

#endif /* COVER_H */
