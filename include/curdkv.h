/*
 * curdkv.h -- C ABI of the CurDKV post-prefill KV selection library for
 * AMD MI355X (gfx950).
 *
 * The library computes Algorithm 1 of "Value-Guided KV Compression for LLMs via
 * Approximated CUR Decomposition" (CurDKV) for every layer and KV group of a
 * GQA cache: sketch, project, row-norm squared, combine, normalise, keep sinks
 * plus top-k, gather.  All arithmetic runs in HIP kernels; there is no CPU
 * fallback.  Layers are an outer batch dimension over the algorithm's group
 * loop; a batch of sequences folds into `layers`.
 *
 * Conventions
 *   - Every function returns CURDKV_OK (0) or a negative error code and never
 *     throws.  Arguments are validated on the host before anything is launched;
 *     on error nothing has been launched.
 *   - "device" pointers are HIP device memory owned by the caller; the library
 *     neither frees nor keeps them.  "host" pointers are ordinary host memory,
 *     read before the call returns.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).  The
 *     compute calls only enqueue work on it and do not synchronise.
 *   - The context owns the sketches, the per-block partial sums, the device
 *     copy of the offsets and the workspaces of the selection and of the budget
 *     allocation, all on the device that was current at curdkv_create;
 *     that device must be current for every later call (else INVALID_ARG).
 *     Calls on one context must not overlap in time on different streams.
 *   - Capturing a compute call in a HIP graph: run the same call (same offsets,
 *     same optional buffers) once and synchronise before the capture, so that
 *     the capture neither uploads offsets nor allocates scratch; both would
 *     make the call unfit for capture.  The captured kernels read the offsets
 *     and the gather's block table from the context's single device copy: as
 *     long as the graph may be replayed, call curdkv_select / curdkv_compact /
 *     curdkv_compress on that context with these same offsets only (or give the
 *     graph a context of its own).  A graph replayed after the copy has changed
 *     would run the captured grid against the new offsets: its results would be
 *     meaningless and, where the new offsets reach further than the captured
 *     buffers, its writes out of bounds: such a graph must not be replayed.
 *     curdkv_compress_adaptive keeps offsets and table in caller buffers and has
 *     no such constraint.
 *   - K and V are row-major [layers, kv_heads, n, head_dim] in the context's
 *     storage type; token j of group (l, h) starts at element
 *     ((l*kv_heads + h)*n + j)*head_dim.  Base pointers must be 16-byte aligned.
 */
#ifndef CURDKV_H
#define CURDKV_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define CURDKV_OK               0
#define CURDKV_ERR_INVALID_ARG -1   /* null pointer, size out of range, inconsistent offsets */
#define CURDKV_ERR_UNSUPPORTED -2   /* head_dim, sketch_dim or dtype the kernels do not cover */
#define CURDKV_ERR_HIP         -3   /* a HIP runtime call failed (no device, launch error, ...) */
#define CURDKV_ERR_OOM         -4   /* device or host allocation failed */
#define CURDKV_ERR_TOO_LARGE   -5   /* more (layer, group) pairs than a non-allocating call's fixed workspace holds */

#define CURDKV_ATTEND_SCRATCH_BYTES 38354944   /* most scratch that an attention call uses (16 KB of counters, 73728 rows of 520 bytes) */

#define CURDKV_DTYPE_F32  0
#define CURDKV_DTYPE_BF16 1

/* What the score of a token is built from.  KV is the method (the combination
 * step of Algorithm 1: product of key and value scores); KEY and VALUE are the
 * ablation of the appendix ("Ablation Study") that uses one tensor alone. */
#define CURDKV_SCORE_KV    0
#define CURDKV_SCORE_KEY   1
#define CURDKV_SCORE_VALUE 2

typedef struct curdkv_ctx curdkv_ctx;

/* Problem statement of Algorithm 1 (inputs K, V in R^{g x n x d}, projection
 * dimension r) extended over layers.  group_size (query heads per KV group)
 * is carried for curdkv_fold; the scores themselves depend on K and V only. */
typedef struct curdkv_config {
    int32_t  layers;       /* >= 1 */
    int32_t  kv_heads;     /* g, number of KV groups per layer, >= 1 */
    int32_t  group_size;   /* query heads per KV group, >= 1 */
    int32_t  head_dim;     /* d; supported: 128 */
    int32_t  sketch_dim;   /* r in [1, 128]; padded internally with zero columns */
    int32_t  dtype;        /* CURDKV_DTYPE_* : storage type of K, V and of G */
    int32_t  score_source; /* CURDKV_SCORE_* ; 0 = the method's key-value product */
    int32_t  no_projection;/* 0 = sketch with G (the method); 1 = the ablation without the Gaussian
                              projection: squared norms of the stored rows */
    int64_t  max_tokens;   /* largest n any call will pass, >= 1 */
    uint64_t seed;         /* seed of the sketch generator */
} curdkv_config;

/* Create a context on the current HIP device: generates the sketch G of every
 * (layer, group) on the host, uploads it in the kernels' operand layout and
 * allocates the workspaces.  Synchronous.  *out is set only on success. */
int curdkv_create(curdkv_ctx** out, const curdkv_config* cfg);

/* Free everything the context owns.  Synchronises the device first.  NULL is accepted. */
int curdkv_destroy(curdkv_ctx* ctx);

/* Host-only (no GPU needed): write G of group (layer, head) to G_host[d*r],
 * row-major [head_dim, sketch_dim], as float.
 *
 * Sampling step of Algorithm 1: a d x r matrix of independent normal entries
 * with variance 1/r; one G per (layer, group), shared by K and V.  The paper fixes no generator:
 * element (i, j) has counter c = ((layer*kv_heads + head)*d + i)*r + j and
 * takes SplitMix64 outputs number 2c+1 and 2c+2 (w1, w2) of the stream started
 * at `seed`; u1 = ((w1>>11)+1)*2^-53, u2 = (w2>>11)*2^-53,
 * G_ij = sqrt(-2 ln u1) cos(2 pi u2) / sqrt(r) in double, then rounded to the
 * storage type (nearest even).  The rounded value is what the kernels use. */
int curdkv_sketch_host(const curdkv_config* cfg, int32_t layer, int32_t head, float* G_host);

/* Replace the sketch of one group by caller-supplied values (host, row-major
 * [head_dim, sketch_dim] floats; rounded to the storage type).  Synchronous.
 * For callers that draw G themselves, as Algorithm 1 literally does. */
int curdkv_set_sketch(curdkv_ctx* ctx, int32_t layer, int32_t head, const float* G_host);

/* Algorithm 1 from the projection step to the normalisation step: for every (layer, group)
 *   lK_j = ||(K G)[j]||^2,  lV_j = ||(V G)[j]||^2,  lKV_j = lK_j * lV_j,
 *   scores_j = lKV_j / sum_j lKV_j   (sum over all n rows; 1/n if the sum is 0).
 * K, V: device, [layers, kv_heads, n, head_dim], storage type, read once.
 * scores: device float [layers, kv_heads, n], written.
 * Products accumulate in fp32; lKV must stay inside the fp32 range.
 * 1 <= n <= max_tokens. */
int curdkv_scores(curdkv_ctx* ctx, const void* K, const void* V, int64_t n,
                  float* scores, void* stream);

/* GQA score fold (Section 2, GQA-compatible eviction; Section 3.2 assumes a
 * group of query heads shares one K_i, V_i): mean over the group of per-query-
 * head scores.  scores_q: device float [layers, kv_heads, group_size, n];
 * scores: device float [layers, kv_heads, n].  CurDKV's own scores are already
 * per group, so the hot path does not need this call; it serves score sources
 * that are per query head.  Summation order is fixed (head 0 first). */
int curdkv_fold(curdkv_ctx* ctx, const float* scores_q, int64_t n, float* scores,
                void* stream);

/* Sink, top-k and union steps of Algorithm 1: S = {0..s-1} U (TopK(scores[s:], k-s) + s)
 * for every (layer, group).
 * scores: device float [layers, kv_heads, n], non-negative, no NaN.
 * budgets: host int32 [layers*kv_heads], k per group (sinks included), 0 <= k <= n.
 * offsets: host int64 [layers*kv_heads + 1], offsets[0] = 0 and
 *          offsets[i+1] = offsets[i] + budgets[i].
 * indices: device int32 [offsets[last]]; group i's tokens go to
 *          indices[offsets[i] .. offsets[i+1]) in ascending token order.
 * Ties: larger score first, then smaller token index.  k <= s keeps tokens
 * 0..k-1.  n_sink >= 0. */
int curdkv_select(curdkv_ctx* ctx, const float* scores, int64_t n,
                  const int32_t* budgets, int32_t n_sink, const int64_t* offsets,
                  int32_t* indices, void* stream);

/* Gather step of Algorithm 1: K' = K[S], V' = V[S] (rows of the original cache).
 * indices, offsets: as written by / passed to curdkv_select (offsets on host;
 * non-decreasing, offsets[0] = 0, each group's count <= n; every index must lie
 * in [0, n)).
 * K_out, V_out: device, packed [offsets[last], head_dim], storage type; equal to
 * [layers, kv_heads, k, head_dim] when all budgets are k.  Bit-exact copies. */
int curdkv_compact(curdkv_ctx* ctx, const void* K, const void* V, int64_t n,
                   const int32_t* indices, const int64_t* offsets,
                   void* K_out, void* V_out, void* stream);

/* The whole of Algorithm 1 in one call: scores, selection and gather, with the
 * results of curdkv_scores + curdkv_select + curdkv_compact (same arguments,
 * same layouts; `scores` may be NULL when the caller does not want them, the
 * library then uses a scratch buffer it allocates on first need).  Where
 * curdkv_uses_fused_kernel says so, one fused kernel does everything with one
 * workgroup per (layer, group) and the scores never pass through HBM between
 * the steps (when more than 11 % of all rows are kept, only its scoring phases
 * are used and the stand-alone selection and gather kernels follow: the gather
 * kernel moves rows faster than the fused kernel's last phase); otherwise
 * the kernels of the separate calls are launched.  The normalising sum is taken
 * in a different order in the two cases, so scores can differ in the last bits
 * between them. */
int curdkv_compress(curdkv_ctx* ctx, const void* K, const void* V, int64_t n,
                    const int32_t* budgets, int32_t n_sink, const int64_t* offsets,
                    float* scores, int32_t* indices, void* K_out, void* V_out, void* stream);

/* Which kernels curdkv_scores / curdkv_compress launch for a cache of n tokens
 * per head: 1 = the fused one-workgroup-per-head kernel, 0 = the general
 * kernels; negative = error code.  The fused kernel needs bf16, a sketch of at
 * most 64 columns (or no projection), n <= 32768, and a number of (layer,
 * group) pairs that fills whole rounds of the GPU's compute units to at least
 * 90 %.  The results are the same either way (Algorithm 1); the entry exists so
 * that tests and tuning know which path they exercise. */
int curdkv_uses_fused_kernel(const curdkv_ctx* ctx, int64_t n);

/* AdaCurDKV head-wise budgets (Section 3.2, "Adaptive budget allocation"): every
 * layer keeps kv_heads*budget tokens in all, the top normalised scores ACROSS the
 * heads of the layer, but each head is guaranteed its own best floor(alpha*budget)
 * tokens (the AdaKV safeguard; the paper uses alpha = 0.20).  Reading: the first
 * s' = min(n_sink, n) tokens of a head are sinks, always kept and counted; each
 * head is guaranteed g = max(floor(alpha*budget) - s', 0) further tokens; the
 * remaining kv_heads*(budget - s' - g) places of a layer go to its largest
 * scores outside the sinks and the guaranteed ones, equal scores in (head, token)
 * order.  budget <= s' gives `budget` to every head.
 * scores: device float [layers, kv_heads, n], normalised, non-negative.
 * budgets_out: DEVICE int32 [layers*kv_heads], tokens to keep per head (sinks
 * included); each layer's entries sum to kv_heads*budget.  Copy them to the host
 * and pass them, with their prefix sums, to curdkv_select and curdkv_compact.
 * 0 <= budget <= n, 0 <= alpha <= 1. */
int curdkv_adaptive_budgets(curdkv_ctx* ctx, const float* scores, int64_t n, int32_t budget,
                            int32_t n_sink, double alpha, int32_t* budgets_out, void* stream);

/* curdkv_adaptive_budgets for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, same results, same kernels; the histograms, key lists and
 * per-layer state that curdkv_adaptive_budgets keeps in a buffer its context got
 * from hipMalloc live here in a static device array of the library (24.5 MiB +
 * 32 KiB per GPU, resident from the moment the library is loaded, its address
 * looked up at curdkv_create).
 * The call makes no hipMalloc, hipFree or other allocating call.
 * Limit: layers*kv_heads <= 1024, else CURDKV_ERR_TOO_LARGE and nothing is launched.
 * All calls on one GPU, from every context, share the one array: two such calls
 * that overlap in time on that GPU race; calls on one stream, or otherwise
 * ordered, are safe (nothing in the array has to survive between calls). */
int curdkv_adaptive_budgets_noalloc(curdkv_ctx* ctx, const float* scores, int64_t n, int32_t budget,
                                    int32_t n_sink, double alpha, int32_t* budgets_out, void* stream);

/* AdaCurDKV in one call with nothing passing through the host (Algorithm 1 with the
 * head-wise budgets of Section 3.2, "Adaptive budget allocation"): scores as in
 * curdkv_scores, budgets as in curdkv_adaptive_budgets, their prefix sums, then the
 * selection and the gather of curdkv_select / curdkv_compact with those budgets,
 * all enqueued on `stream` without a synchronisation or a copy to the host.
 * Every layer keeps kv_heads*budget rows, so the sizes are known beforehand:
 * scores: device float [layers, kv_heads, n], or NULL (library scratch, allocated
 *   on first need);
 * budgets_out: device int32 [layers*kv_heads]; offsets_out: device int64
 *   [layers*kv_heads + 1], offsets_out[i] = budgets_out[0] + .. + budgets_out[i-1];
 * indices: device int32 [layers*kv_heads*budget]; K_out, V_out: device
 *   [layers*kv_heads*budget, head_dim]; group i owns rows offsets_out[i] ..
 *   offsets_out[i+1]-1 of all three, tokens ascending.
 * 0 <= budget <= n, 0 <= alpha <= 1, n_sink >= 0; kv_heads <= 1024. */
int curdkv_compress_adaptive(curdkv_ctx* ctx, const void* K, const void* V, int64_t n,
                             int32_t budget, int32_t n_sink, double alpha, float* scores,
                             int32_t* budgets_out, int64_t* offsets_out, int32_t* indices,
                             void* K_out, void* V_out, void* stream);

/* Scoring during generation (Section 3.2, first paragraph: the method is meant for
 * the generation phase as well as for pre-filling).  The un-normalised scores
 * lKV_j of a token do not depend on the other tokens, so a growing cache is scored
 * chunk by chunk: this call scores the m new tokens of every (layer, group),
 * writes lKV to raw[group*stride + n_old + j] and adds their sum to sums[group]
 * (n_old == 0 starts the sums afresh).
 * K_new, V_new: device, [layers, kv_heads, m, head_dim], the new rows only.
 * raw: device float [layers*kv_heads, stride]; sums: device double [layers*kv_heads].
 * 1 <= m, 0 <= n_old, n_old + m <= stride <= max_tokens. */
int curdkv_scores_append(curdkv_ctx* ctx, const void* K_new, const void* V_new, int64_t m,
                         int64_t n_old, int64_t stride, float* raw, double* sums, void* stream);

/* Normalisation step for the first n tokens of a cache scored with curdkv_scores_append:
 * scores[group*n + j] = raw[group*stride + j] / sums[group] (1/n if the sum is 0),
 * sums being those of exactly these n tokens.  The result is what curdkv_scores
 * gives on the n-token cache (up to the order of the additions in the sum) and
 * goes to curdkv_select / curdkv_adaptive_budgets. */
int curdkv_normalise(curdkv_ctx* ctx, const float* raw, const double* sums, int64_t stride,
                     int64_t n, float* scores, void* stream);

/* ---- around a compressed cache: its rows made, attended to, and held in 4 bits ----
 *
 * These calls take one layer at a time: `count` sequences of that layer, kv_heads,
 * group_size, head_dim and dtype those of the context (its layers, sketches and seed play
 * no part).  A layer's cache is [count, kv_heads, stride, head_dim] in the storage type:
 * row j of head h of sequence b starts at element ((b*kv_heads + h)*stride + j)*head_dim
 * (a contiguous cache of n tokens, as the calls above take it, has stride = n).  Queries
 * and results are token-major, [count, m, kv_heads*group_size, head_dim], query head
 * h*group_size + i belonging to KV head h.  Device pointers to rows, codes and tables are
 * 16-byte aligned.  Arrays of lengths, rows and positions are device memory and are not
 * looked at on the host: what lies outside the stated ranges is clamped or left out as
 * said, and nothing is read or written outside the buffers. */

/* Norms of queries and keys for each head, their rotation by position, and the new rows of
 * the cache, from a layer's projections.
 * qkv: device, count*m rows of (group_size + 2)*kv_heads heads of head_dim values in the
 *   storage type: queries, then keys, then values; row_stride elements from one row to the
 *   next (at least (group_size + 2)*kv_heads*head_dim, a multiple of 16 bytes).  Row b*m + i
 *   is token i of sequence b.
 * starts: int32 [count], the cache row of a sequence's first new token; NULL = 0.  Tokens
 *   whose row lies outside [0, stride) leave the cache as it is.
 * positions: int32 [count*m]; NULL = the token's cache row.  Clamped to [0, table_rows).
 * table: float [table_rows, 2, head_dim/2]: cosines, then sines, of a position's angles.
 * q_weight, k_weight: storage type [head_dim]: y = x / sqrt(mean(x^2) + eps) * weight
 *   before the rotation; NULL = no norm of queries / of keys.
 * pairs: 0: channels i and head_dim/2 + i turn together, 1: channels 2i and 2i + 1, by
 *   (a, b) -> (a cos - b sin, b cos + a sin) of angle i.
 * Q: written [count, m, kv_heads*group_size, head_dim]; K, V: the layer's cache, of which
 *   the new tokens' rows are written (values as they are).  Nothing may overlap qkv.
 * 32 bits throughout, rounded once at the store.  stride <= max_tokens. */
int curdkv_rotate(curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride,
                  const int32_t* starts, const int32_t* positions, const float* table,
                  int64_t table_rows, const void* q_weight, const void* k_weight, float eps,
                  int32_t pairs, void* Q, void* K, void* V, int64_t stride, void* stream);

/* Causal attention of each sequence's last m tokens over its cache, with an optional window
 * and first tokens that stay visible: of a sequence of `length` tokens, new token i stands at
 * position p = length - m + i and sees row j where j <= p and (window == 0 or p - j < window
 * or j < n_sink);
 *   out = sum_j softmax_j(scale * q.k_j) v_j,  lse = log sum_j exp(scale * q.k_j).
 * A token that sees nothing (length < m and i < m - length), or only keys whose scores are
 * -infinity, gets zeros and -infinity; a key of such a score weighs nothing.  What a token does
 * not see does not reach it, infinities and NaN included.  A score of +infinity or NaN that it
 * sees makes its result and lse NaN, and a value that is not finite makes its channel so,
 * whatever the key weighs.
 * lengths: int32 [count], clamped to [0, n]; NULL = n for all.  n <= stride, n <= max_tokens.
 * count*m*kv_heads*group_size < 2^31, and m*kv_heads*group_size < 2^28 where 16 queries of a KV head
 * make a workgroup (few tokens; fp32 and 4-bit kept rows); else CURDKV_ERR_UNSUPPORTED.
 * out as Q; lse: float [count, kv_heads*group_size, m] or NULL.  scale > 0; m <= max_tokens.
 * m = n is a prompt, m = 1 a generated token; scores, weights' sum and results are held in 32 bits;
 * with a bf16 cache the weights are rounded to bf16 for their product with V; with an fp32 cache
 * every product is good to 2^-22 of itself, or to 2^-133 of its larger factor where that is more.
 * Sums of values times weights of up to 2^8 are divided by the weights' sum at the end: values of
 * magnitude 2^120 / n and more may pass the range of 32 bits on the way.
 * scratch: device memory of the caller's, 16-byte aligned, for the partial results of few tokens over
 *   long caches, whose heads are shared out over many workgroups; CURDKV_ATTEND_SCRATCH_BYTES
 *   are as much as a call ever uses, with less (0 and NULL included) there are fewer shares.
 *   It is cleared (zeros) once, before the first call that it is given to; every call leaves its counters
 *   cleared.  Calls that overlap in time need one each. */
int curdkv_attend(curdkv_ctx* ctx, const void* Q, const void* K, const void* V, int64_t count,
                  int64_t m, int64_t n, int64_t stride, const int32_t* lengths, int64_t window,
                  int32_t n_sink, float scale, void* out, float* lse, void* scratch,
                  int64_t scratch_bytes, void* stream);

/* The gather of curdkv_compact into 4 bits (the open microscaling format MXFP4): blocks of 32
 * channels share a power of two 2^e, e = floor(log2(largest magnitude)) - 2, at least -127,
 * and a value x is held as the nearest to x/2^e of 0, .5, 1, 1.5, 2, 3, 4, 6 with its sign (ties
 * to the even code, beyond 6 to 6).  A block that holds an infinity or NaN stands for NaN.
 * K, V, n, indices: as curdkv_compact takes them; offsets: the same, but in DEVICE memory
 *   (curdkv_compress_adaptive leaves them there), and total = offsets[last], at most
 *   layers*kv_heads*n.  An index outside [0, n) leaves its row unwritten.
 * K_codes, V_codes: [offsets[last], head_dim/2], channel 2i in the low half of byte i;
 * K_scales, V_scales: [offsets[last], head_dim/32], e + 127, or 255 for NaN. */
int curdkv_compact_mx(curdkv_ctx* ctx, const void* K, const void* V, int64_t n,
                      const int32_t* indices, const int64_t* offsets, int64_t total, uint8_t* K_codes,
                      uint8_t* K_scales, uint8_t* V_codes, uint8_t* V_scales, void* stream);

/* The values that rows in 4 bits stand for, in the storage type (exact; NaN where a scale is 255, whatever
 * the codes): out [rows, head_dim]. */
int curdkv_expand_mx(curdkv_ctx* ctx, const uint8_t* codes, const uint8_t* scales, int64_t rows,
                     void* out, void* stream);

/* Attention of m new tokens over the rows that a selection kept and over the tokens since:
 * every new token sees all kept rows of its head, and, causally, the tail: of `length` tail
 * tokens, new token i stands at p = length - m + i and sees tail rows j <= p (the new tokens'
 * own rows are part of the tail).  out, lse, scale and scratch as in curdkv_attend.
 * K_kept, V_kept: packed rows as the gathers write them; those of KV head h of sequence b are rows
 *   offsets[b*kv_heads + h] .. offsets[b*kv_heads + h + 1] - 1.
 * offsets: DEVICE int64 [count*kv_heads + 1], kept within [0, total]; a layer of a larger
 *   packed cache is its slice of the offsets, with the whole cache's K_kept and V_kept.
 * total: rows of K_kept and V_kept, below 2^31; rows: how many of them belong to this call's heads (all:
 *   total).  The work is shared out by their average; uneven heads are read whole all the same.
 * K_tail, V_tail: [count, kv_heads, tail_stride, head_dim]; tail_lengths: int32 [count], clamped
 *   to [0, tail_n]; NULL = tail_n.  tail_n = 0: no tail (the pointers may be NULL). */
int curdkv_attend_kept(curdkv_ctx* ctx, const void* Q, const void* K_kept, const void* V_kept,
                       const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail,
                       const void* V_tail, int64_t tail_n, int64_t tail_stride, const int32_t* tail_lengths,
                       int64_t count, int64_t m, float scale, void* out, float* lse, void* scratch,
                       int64_t scratch_bytes, void* stream);

/* The same over kept rows held in 4 bits (curdkv_compact_mx); the tail is in the storage type. */
int curdkv_attend_kept_mx(curdkv_ctx* ctx, const void* Q, const uint8_t* K_codes,
                          const uint8_t* K_scales, const uint8_t* V_codes, const uint8_t* V_scales,
                          const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail,
                          const void* V_tail, int64_t tail_n, int64_t tail_stride,
                          const int32_t* tail_lengths, int64_t count, int64_t m, float scale,
                          void* out, float* lse, void* scratch, int64_t scratch_bytes, void* stream);

/* ---- a cache that stays at its size, and one that serves several answers ----
 *
 * These calls, too, take one layer at a time, with the conventions of those above. */

/* curdkv_rotate where a token stands at several positions, as time, height and width of a video's patch: each
 * of the head_dim/2 angles turns by the position on its own axis.
 * axis_of: HOST uint8 [head_dim/2], the axis of every angle, below `axes` (1 to 4).
 * positions: int32 [axes, count*m], not NULL; each clamped to [0, table_rows).  All else as curdkv_rotate, which this
 *   is, bit for bit, where a token's positions are the same on all axes. */
int curdkv_rotate_axes(curdkv_ctx* ctx, const void* qkv, int64_t count, int64_t m, int64_t row_stride,
                       const int32_t* starts, const int32_t* positions, int32_t axes, const uint8_t* axis_of,
                       const float* table, int64_t table_rows, const void* q_weight, const void* k_weight, float eps,
                       int32_t pairs, void* Q, void* K, void* V, int64_t stride, void* stream);

/* The attention weight that every cached key got from each sequence's last m tokens, over the group_size query
 * heads of its KV head, added to what is left of the weight that it had:
 *   mass[b, h, j] = decay * mass[b, h, j] + sum_i sum_t exp(scale * q_ti.k_j - lse[b, h*group_size + i, t])
 * over the query heads i of KV head h and the tokens t that see key j (as in curdkv_attend: causal, window, n_sink).
 * A whole prompt's weights are m = n; those that its last tokens give it (an observation window) fewer; a
 * generated token's m = 1.
 * Q, K, count, m, n, stride, lengths, window, n_sink, scale: as curdkv_attend takes them; lse: float [count,
 *   kv_heads*group_size, m], what curdkv_attend wrote for them.  A token of lse -infinity (it sees nothing,
 *   or is left out, as padding) gives nothing to any key, whatever its queries and the keys hold; one of lse NaN makes the
 *   weight of the keys that it sees NaN, and no other's.
 * decay: not negative, finite; 0: the old weights are not read.
 * kv_heads <= 16384, kv_heads*group_size <= 2^20, ceil(n/64)*count*kv_heads < 2^24.
 * mass: float [count, kv_heads, mass_stride], rows below a sequence's length written; those behind it stay as they
 *   are.  n <= mass_stride.
 * Scores and sums in 32 bits, summed in an order that the sizes, lengths, window, scratch_bytes and the device's number of
 * compute units give, and nothing else: the same call gives the same bits.  scratch as in curdkv_attend. */
int curdkv_attend_weights(curdkv_ctx* ctx, const void* Q, const void* K, const float* lse, int64_t count,
                          int64_t m, int64_t n, int64_t stride, const int32_t* lengths, int64_t window, int32_t n_sink,
                          float scale, float decay, float* mass, int64_t mass_stride, void* scratch,
                          int64_t scratch_bytes, void* stream);

/* Eviction by accumulated weight: of each head's rows (a sequence's `length`) `keep` stay, or all where there are no more.
 * First those whose position is below n_sink or among the `recent` last ones (above the head's largest position less
 * `recent`), then those of the largest mass (NaN above all, -0 as 0), of equal ones the lower row.  Should the first be more
 * than `keep`, the mass decides among them.  n_sink + recent <= keep.
 * A row below `keep` that stays keeps its place; the places of the others are taken, in ascending order, by the rows that
 * stay from beyond, ascending: rows are no longer in the order of their tokens, and `positions` says which is which.
 * K, V: [count, kv_heads, stride, head_dim]; mass: float, positions: int32 [count, kv_heads, stride]; positions NULL: the
 *   row's number.  lengths: int32 [count], clamped to [0, n]; NULL = n.  1 <= keep <= 2^30, n <= stride, n <= 524288,
 *   count*kv_heads <= 2^20.
 * K_out, V_out: [count, kv_heads, out_stride, head_dim]; mass_out, positions_out: [count, kv_heads, out_stride], NULL: not
 *   written.  Only rows below min(length, keep) are written.  keep <= out_stride or n <= out_stride.
 *   K_out = K with V_out = V: in place, and mass_out may be mass, positions_out positions; wherever an array is its own
 *   output, out_stride = stride.  Nothing else may overlap.
 * rows: int32 [count, kv_heads, keep], written: the row that each place's row came from; -1 beyond min(length, keep). */
int curdkv_evict(curdkv_ctx* ctx, const void* K, const void* V, const float* mass, const int32_t* positions,
                 int64_t count, int64_t n, int64_t stride, const int32_t* lengths, int64_t keep, int32_t n_sink,
                 int64_t recent, void* K_out, void* V_out, float* mass_out, int32_t* positions_out, int64_t out_stride,
                 int32_t* rows, void* stream);

/* curdkv_attend_kept for sequences that share their kept rows: `share` of them follow each of `count` prefixes, whose rows
 * are read once for all.  Sequence b*share + s of the count*share sequences sees the kept rows of prefix b and, causally,
 * its own tail.
 * Q, out: [count*share, m, kv_heads*group_size, head_dim]; lse: float [count*share, kv_heads*group_size, m] or NULL.
 * offsets: DEVICE int64 [count*kv_heads + 1], K_kept, V_kept, total, rows: the prefixes', as in curdkv_attend_kept.
 * K_tail, V_tail: [count*share, kv_heads, tail_stride, head_dim]; tail_lengths: int32 [count*share].
 * count*share*m*kv_heads*group_size < 2^31, kv_heads*group_size <= 16384, kv_heads <= 1024.  scratch: not NULL here,
 * CURDKV_ATTEND_SCRATCH_BYTES at least, cleared once as for curdkv_attend; the partial results of prefixes and tails meet
 * there.
 * The kept rows are shared out over the device, a tail is not: one workgroup reads all of a sequence's KV head.  It is made
 * for tails that are short beside the prefix; where a few sequences have thousands of tokens of their own,
 * curdkv_attend_kept, which shares tails out too, is the faster call (and needs the kept rows once for every sequence). */
int curdkv_attend_shared(curdkv_ctx* ctx, const void* Q, const void* K_kept, const void* V_kept,
                         const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail,
                         const void* V_tail, int64_t tail_n, int64_t tail_stride, const int32_t* tail_lengths,
                         int64_t count, int64_t share, int64_t m, float scale, void* out, float* lse, void* scratch,
                         int64_t scratch_bytes, void* stream);

/* The same over kept rows held in 4 bits (curdkv_compact_mx); the tails are in the storage type. */
int curdkv_attend_shared_mx(curdkv_ctx* ctx, const void* Q, const uint8_t* K_codes,
                            const uint8_t* K_scales, const uint8_t* V_codes, const uint8_t* V_scales,
                            const int64_t* offsets, int64_t total, int64_t rows, const void* K_tail,
                            const void* V_tail, int64_t tail_n, int64_t tail_stride, const int32_t* tail_lengths,
                            int64_t count, int64_t share, int64_t m, float scale, void* out, float* lse, void* scratch,
                            int64_t scratch_bytes, void* stream);

/* Text for an error code; never NULL. */
const char* curdkv_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* CURDKV_H */
