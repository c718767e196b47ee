/*
 * pbs.h -- C ABI of the MI355X-native PBS-Attn prefill path.
 *
 * PBS-Attn = Permuted Block-Sparse Attention (arXiv 2510.21270).  One prefill
 * attention forward pass is Algorithm 1 of the paper:
 *
 *   pbs_key_scores      Eq. 4   global importance score of every key
 *   pbs_segment_permute Eq. 5   per-segment descending argsort + K', V' = P_pi K, P_pi V
 *   pbs_block_mask      Alg. 2  mean-pooled cumulative-mass block selection on (Q', K')
 *   pbs_attn_fwd        Alg. 1  online-softmax attention over the selected blocks only
 *   pbs_unpermute       Alg. 1  O = P_sigma^T O'   (Theorem 1)
 *
 * General conventions
 *   - Every tensor pointer is a DEVICE pointer to caller-owned, contiguous,
 *     row-major memory, 16-byte aligned.  The library never allocates, frees
 *     or synchronises; all work is enqueued on `stream` (a hipStream_t passed
 *     as void*, NULL = the default stream) and is complete when the stream is.
 *   - `pbs_problem` itself is a HOST pointer and is read during the call only.
 *   - Arguments are validated on the host before anything is launched; a bad
 *     call returns a status and enqueues nothing.  A failed launch returns
 *     PBS_ERR_HIP.  Nothing throws or aborts.
 *   - Q is [batch, h_q, n, d]; K and V are [batch, h_kv, n, d]; h_q % h_kv == 0
 *     and query head h reads kv head h / (h_q / h_kv)  (grouped-query attention;
 *     one permutation per kv head, the "shared permutation strategy" of the
 *     appendix "GQA Handling"; the replicated default of the paper is the case
 *     h_kv == h_q).
 *   - T = ceil(n / block) blocks; segment % block == 0; R = segment / block;
 *     G = floor(n / segment) full segments; tokens at or beyond G * segment are
 *     never permuted (Section "Segmented Permutation for Causal Attention").
 *   - Index vectors are in gather form with absolute positions: slot p of a
 *     permuted tensor holds original token idx[p], and idx maps every segment
 *     onto itself.
 *   - K' ("Kp") keeps the [batch, h_kv, n, d] layout.  V' is kept as "Vt":
 *     [batch, h_kv, T, block / G, d, G] with G = min(block, 32), i.e. every
 *     key block stored as groups of G consecutive key slots, each group
 *     transposed (feature-major), the slots past n in the last block
 *     zero-filled.  Vt is produced by pbs_segment_permute and consumed by
 *     pbs_attn_fwd; pbs_vt_bytes gives its size.
 *   - Supported: dtype PBS_BF16 or PBS_F32; d in {64, 128}; block in
 *     {16, 32, 64, 128}; segment <= 4096; T <= 4096; any n >= 1.  Attention over PBS_BF16 with block in {64, 128} runs
 *     on the bf16 matrix cores (d = 64 with fp32 probabilities, each in three bf16 terms); every other supported
 *     combination in fp32 arithmetic.
 *   - Results are deterministic: the same inputs give bit-identical outputs.
 */
#ifndef PBS_H
#define PBS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PBS_OK = 0,
    PBS_ERR_NULL = 1,        /* a required pointer is NULL */
    PBS_ERR_SHAPE = 2,       /* inconsistent sizes (h_q % h_kv, segment % block, n < 1, ...) */
    PBS_ERR_UNSUPPORTED = 3, /* valid problem outside the supported set listed above */
    PBS_ERR_WORKSPACE = 4,   /* ws_bytes smaller than pbs_workspace_bytes(), or ws misaligned */
    PBS_ERR_HIP = 5          /* a kernel launch failed */
} pbs_status;

/* PBS_E4M3 (8-bit floating point, 4 exponent and 3 mantissa bits, no infinities) and PBS_I8 are types of a pbs_cache only. */
typedef enum { PBS_F32 = 0, PBS_BF16 = 1, PBS_E4M3 = 2, PBS_I8 = 3 } pbs_dtype;

/*
 * PBS_FLAG_FORCE_FIRST_BLOCK: Algorithm 2 also keeps key block 0 in every row.
 * PBS_FLAG_TOKEN_ORDER_COPY: K', Vt and kidx each carry a second tensor of the same shape in token order (K
 *   itself, V block-transposed without permutation, kidx = 0 .. n-1) in the same allocation, starting
 *   batch * h_kv * T * block rows (K': rows of d elements; kidx: entries; Vt: key slots of d elements, i.e. directly
 *   behind the first tensor) after the start of the permuted one; each buffer therefore holds
 *   batch * h_kv * (T * block + n) rows (Vt: 2 * batch * h_kv * T * block).  pbs_segment_permute writes both; every
 *   other stage reads the first tensor as before, and pbs_attn_fwd may evaluate a query block's own segment from
 *   the second (see there).  The result is the same attention: the order in which keys are summed does not matter
 *   (Theorem 1).
 * PBS_FLAG_RUNNING_MAX_ONLY: pbs_attn_fwd evaluates every query block with the running-maximum recurrence of
 *   Algorithm 1 as printed (m moves and O, l are rescaled); for bf16, d = 128, block = 128 this leaves out the first
 *   pass, which keeps a fixed softmax reference per query.  Same result up to rounding; slower.
 * PBS_FLAG_KBAR_IN_WS: the workspace given to pbs_block_mask already holds the block means of Kp, left there by
 *   the pbs_segment_permute call that wrote this Kp (see its `ws`); pbs_block_mask then does not read Kp at all.
 * PBS_FLAG_INDEX_REMAP: index remapping as the appendix "Memory Overhead" sketches it (the attention kernel retrieves
 *   the keys from the original tensor through the permuted indices): no K' exists.  pbs_segment_permute writes kidx
 *   and Vt only (its Kp argument is ignored and may be NULL; with a workspace it still leaves the block means of the
 *   permuted keys there), pbs_block_mask must then be given PBS_FLAG_KBAR_IN_WS as well, and pbs_attn_fwd takes the
 *   caller's K in place of Kp and gathers the rows kidx[slot] while it stages its tiles.  bf16, d = 128, block 64 or
 *   128 only (PBS_ERR_UNSUPPORTED otherwise, and together with PBS_FLAG_TOKEN_ORDER_COPY); same results as with a
 *   materialised K', bit for bit against PBS_FLAG_RUNNING_MAX_ONLY (it runs on that kernel).  V' stays materialised
 *   as Vt: the second matrix product needs it feature-major.
 */
enum { PBS_FLAG_FORCE_FIRST_BLOCK = 1u, PBS_FLAG_TOKEN_ORDER_COPY = 2u, PBS_FLAG_RUNNING_MAX_ONLY = 4u,
       PBS_FLAG_KBAR_IN_WS = 8u, PBS_FLAG_INDEX_REMAP = 16u };

typedef enum {
    PBS_STAGE_KEY_SCORES = 1,
    PBS_STAGE_SEGMENT_PERMUTE = 2,
    PBS_STAGE_BLOCK_MASK = 3,
    PBS_STAGE_ATTN_FWD = 4,
    PBS_STAGE_UNPERMUTE = 5,
    PBS_STAGE_QUERY_PERMUTE = 6   /* pbs_query_permutation, an ablation outside Algorithm 1's main setting */
} pbs_stage;

typedef struct {
    int32_t batch, h_q, h_kv, n, d;
    int32_t block;    /* B of the paper */
    int32_t segment;  /* S of the paper */
    int32_t dtype;    /* pbs_dtype of Q, K, V, K', Vt, O', O */
    float tau;        /* mass threshold of Alg. 2, compared as (double)tau */
    float scale;      /* logit scale; 0 means 1/sqrt(d) (formed in double where the arithmetic is fp64) */
    uint32_t flags;   /* PBS_FLAG_* */
} pbs_problem;

/* Static string for a status code (never NULL). */
const char *pbs_status_string(pbs_status st);

/* PBS_OK when the problem is inside the supported set, else the status every stage would return. */
pbs_status pbs_validate(const pbs_problem *p);

/* Bytes of scratch a stage needs in `ws` (256-byte aligned device memory); 0 for an invalid problem. */
size_t pbs_workspace_bytes(const pbs_problem *p, int stage);

/* Bytes of the Vt tensor: batch * h_kv * T * d * block elements of the problem's dtype, twice that with
 * PBS_FLAG_TOKEN_ORDER_COPY. */
size_t pbs_vt_bytes(const pbs_problem *p);

/*
 * Eq. 4, with the queries of a GQA group averaged (appendix "GQA Handling"):
 *   Qhat = mean over the group's query heads of the last min(block, n) rows of Q,
 *   scores = mean_rows( softmax_over_all_n_keys( Qhat K^T * scale ) ).
 * No causal mask (Eq. 4 has none).  Q [batch,h_q,n,d] (only the last rows are read), K [batch,h_kv,n,d]
 * -> scores [batch,h_kv,n] float32.  bf16 inputs: matrix cores with an fp32 accumulator and a two-term
 * split of Qhat; fp32 inputs: fp64 accumulation.
 */
pbs_status pbs_key_scores(const pbs_problem *p, const void *Q, const void *K, float *scores,
                          void *ws, size_t ws_bytes, void *stream);

/*
 * The other proxies for the importance score that the paper ablates (Section "The Problem of Information
 * Fragmentation", heuristic 4; appendix "Task-wise Proxy Sensitivity"): the formula of Eq. 4 with another set of
 * query rows standing for all queries.
 *   PBS_PROXY_LAST_BLOCK   the last min(block, n) rows: exactly pbs_key_scores (Last-Block-Query-Attn).
 *   PBS_PROXY_QUERY_ROWS   the m rows at the positions qrows[0 .. m-1] (device memory, int32, the same positions for
 *                          every head; 1 <= m <= 128; a position outside [0, n) is clamped into it; a position listed
 *                          twice counts twice).  With positions drawn at random by the caller: Random-Query-Attn.
 *   PBS_PROXY_AVG_QUERY    one query: the mean over all n positions of the group-averaged query vectors (the reading
 *                          taken of Avg-Query-Attn, which the paper only names); Q is read in full.
 * No causal mask, as in Eq. 4.  Arguments, workspace and precision otherwise as pbs_key_scores.
 * Errors: as pbs_key_scores, plus PBS_ERR_UNSUPPORTED for an unknown proxy, PBS_ERR_NULL / PBS_ERR_SHAPE for a
 * missing qrows / an m outside [1, 128].
 */
typedef enum { PBS_PROXY_LAST_BLOCK = 0, PBS_PROXY_QUERY_ROWS = 1, PBS_PROXY_AVG_QUERY = 2 } pbs_proxy;
pbs_status pbs_key_scores_proxy(const pbs_problem *p, int proxy, const int32_t *qrows, int32_t m, const void *Q,
                                const void *K, float *scores, void *ws, size_t ws_bytes, void *stream);

/*
 * For callers that cannot allocate or pass scratch memory (code under HIP graph capture that owns no workspace,
 * tight serving loops, harnesses that forbid hipMalloc): pbs_key_scores with its scratch memory in a device array
 * that is part of the library image instead of in `ws`.  Same arguments otherwise, same kernels, bit-identical
 * scores.  Allocates nothing and calls no allocating routine.
 *   The array holds pbs_key_scores_static_scratch_bytes() = 4 MiB on every GPU the library runs on, until the
 *   process ends; a problem whose pbs_workspace_bytes(p, PBS_STAGE_KEY_SCORES) is larger is rejected with
 *   PBS_ERR_WORKSPACE and nothing is enqueued (the headline layer, 8 kv heads x 131072 keys, needs 2.6 MiB).
 *   All calls on one GPU share that GPU's array: two calls whose kernels may overlap in time (different streams,
 *   or different host threads without ordering between their streams) race on it; calls on one stream are safe.
 *   Nothing in the array has to be cleared between calls: every word that a call reads it has written before.
 * Errors: as pbs_key_scores, plus PBS_ERR_HIP when the array's address cannot be obtained on the current device.
 */
pbs_status pbs_key_scores_static(const pbs_problem *p, const void *Q, const void *K, float *scores, void *stream);
size_t pbs_key_scores_static_scratch_bytes(void);

/*
 * Eq. 5 inside each full segment: kidx[g*S + t] = g*S + (position of the t-th largest score of segment g),
 * equal scores in ascending position (stable), tail positions kept (identity).  Then Algorithm 1's first
 * step for keys and values: Kp[slot] = K[kidx[slot]], Vt = block-transposed V[kidx[.]].
 *   scores [batch,h_kv,n] float32, or NULL for the identity permutation (the unpermuted MeanPooling
 *     baseline of the appendix "Block Selection in PBS-Attn": K' = K, V' = V).  NaN scores are not supported.
 *   kidx   [batch,h_kv,n] int32, written.
 *   Kp, Vt written; pass both NULL to compute kidx only (K and V may then be NULL too).
 *   ws: optional.  NULL: nothing more.  Otherwise at least pbs_workspace_bytes(p, PBS_STAGE_BLOCK_MASK) bytes,
 *   256-byte aligned (else PBS_ERR_WORKSPACE): the block means of K' that Algorithm 2 starts from are written there
 *   while K' is gathered (the first step of pbs_block_mask moved up one stage, so that K' is not read again for it);
 *   hand the same memory to pbs_block_mask with PBS_FLAG_KBAR_IN_WS set.  Ignored when Kp is NULL.
 */
pbs_status pbs_segment_permute(const pbs_problem *p, const float *scores, const void *K, const void *V,
                               int32_t *kidx, void *Kp, void *Vt, void *ws, size_t ws_bytes, void *stream);

/*
 * Algorithm 1's first step for any [batch, heads, n, d] tensor: Xp[slot] = X[idx[slot]] (Q' = P_sigma Q for a
 * caller-supplied segment-wise sigma; the paper's main setting P_sigma = I needs no call).
 * idx [batch,heads,n] int32 with values in [0, n); an out-of-range entry yields a zero row.
 */
pbs_status pbs_permute_rows(const pbs_problem *p, int32_t heads, const void *X, const int32_t *idx, void *Xp,
                            void *stream);

/*
 * Key-aware query permutation, the ablation of Section "Design Choice: Why Permute Keys but not Queries?" (the
 * paper's main setting keeps P_sigma = I and needs no call).  Centroids Kbar_j = block means of Kc (the keys the
 * queries will attend to: K, or K' when the keys are permuted first; valid rows only in a partial last block).  Every
 * query of a full segment g is assigned to the centroid of highest cosine similarity among those its segment may see,
 * j < (g+1)*R capped at T, ties to the lowest j; sigma orders the queries of the segment by assigned centroid,
 * ascending, queries of one centroid in their original order; tokens past the last full segment keep their place.
 * ("Assigned greedily" is read as: every query takes its single best centroid, no capacity, no reassignment.)
 *   Q [batch,h_q,n,d]; Kc [batch,h_kv,n,d]; qidx [batch,h_q,n] int32 written, gather form with absolute positions:
 *   Q'[slot] = Q[qidx[slot]] (pbs_permute_rows), O[qidx[slot]] = O'[slot] (pbs_unpermute).
 *   ws: pbs_workspace_bytes(p, PBS_STAGE_QUERY_PERMUTE) bytes.  IEEE fp64, features in ascending order, separate
 *   multiplications and additions: the assignment does not depend on the machine.
 * Errors: PBS_ERR_NULL, PBS_ERR_SHAPE (misaligned), PBS_ERR_WORKSPACE, the statuses of pbs_validate, PBS_ERR_HIP.
 */
pbs_status pbs_query_permutation(const pbs_problem *p, const void *Q, const void *Kc, int32_t *qidx, void *ws,
                                 size_t ws_bytes, void *stream);

/*
 * Algorithm 2 on the permuted (Q', K'), per query head:
 *   block means (valid rows only in a partial last block);
 *   a_i = softmax_j(Qbar_i . Kbar_j * scale) over the columns the extended causal mask C admits:
 *         j < (g(i)+1)*R for a query block inside full segment g(i), j <= i past the last full segment;
 *   stable descending sort (ties: lowest j), cumulative sum, k = min({t : c[t] >= tau} U {n_i}), first k kept.
 * All of this is IEEE fp64 in the order of the definition (block means: rows ascending for fp32 storage; for bf16
 * storage any order gives the exact sum; logits: features ascending), so that the discrete result does not depend
 * on how a machine rounds lower precision.  Where the evaluation differs from a plain left-to-right one with
 * separate multiplications and additions, it does so by single roundings: the logits use fused multiply-adds (the
 * same bits whenever the products are exact, as they are for block means of bf16 values unless one column of a block
 * spreads over more than about ten binades), and two sums are formed in a tree order (the softmax denominator and
 * the partial masses the threshold search compares with tau).  A selection can then differ from the plain
 * evaluation only if a cumulative mass lies within a few 1e-16 of tau.  Then the blocks of the
 * query block's own segment are switched on (Section "Effect of Segment Size": they cannot be skipped); past the
 * last full segment only the diagonal block; and block 0 when PBS_FLAG_FORCE_FIRST_BLOCK is set (Section
 * "Baselines").  Forced blocks do not change k.
 *   mask_bits [batch,h_q,T,ceil(T/64)] uint64, bit (j & 63) of word (j >> 6) of row i = M[i][j];
 *   row_cnt   [batch,h_q,T] int32; col_idx [batch,h_q,T,T] int32, the first row_cnt[i] entries of row i are the
 *   selected j ascending, the rest is left untouched.
 */
pbs_status pbs_block_mask(const pbs_problem *p, const void *Qp, const void *Kp, uint64_t *mask_bits,
                          int32_t *row_cnt, int32_t *col_idx, void *ws, size_t ws_bytes, void *stream);

/*
 * Algorithm 1's main loop: for every query block i, over the listed key blocks only (a block that is not
 * listed leaves the running (O, m, l) untouched): S = Q'_i K'_j^T * scale, online softmax, O'_i = diag(l)^-1 O.
 * Inside the query block's own segment, and in the unpermuted tail, entry (row, col) takes part only if the
 * key's original position is not after the query's: kidx[j*block+col] <= qidx[i*block+row]; key slots >= n never
 * take part.  Listed blocks outside the columns C admits are ignored.  A query row that sees no key at all gets
 * a zero output row and lse = -inf (cannot happen when the diagonal block is listed).
 *   Qp [batch,h_q,n,d]; Kp [batch,h_kv,n,d]; Vt as above; qidx [batch,h_q,n] or NULL (identity);
 *   kidx [batch,h_kv,n]; row_cnt, col_idx as written by pbs_block_mask (any order of the listed blocks is
 *   accepted); Op [batch,h_q,n,d] written; lse [batch,h_q,n] float32 or NULL: log-sum-exp of the visible,
 *   listed logits of every query row.
 *   ws: pbs_workspace_bytes(p, PBS_STAGE_ATTN_FWD) bytes, 256-byte aligned device memory (0 bytes, and ws may be NULL,
 *   unless dtype is bf16 with d = 128 and block = 128).  For that shape the call launches up to three kernels on the
 *   stream: one that takes a set of row queues from the library's pool (problems of 4096 query blocks and more; the next
 *   kernel gives it back), one that keeps a fixed softmax reference per query and writes one flag per query block into
 *   ws (not 0 = some probability outgrew the reference by more than 2^64), and one that recomputes the flagged query
 *   blocks with the running-maximum recurrence of Algorithm 1.  The contents of ws need not be initialised and mean
 *   nothing afterwards.
 *   With PBS_FLAG_RUNNING_MAX_ONLY every query block of that shape goes through the second kernel alone.
 *   With PBS_FLAG_TOKEN_ORDER_COPY (Kp, Vt, kidx carry their token-order copies), qidx == NULL and that same shape, a
 *   query block inside a full segment whose list ends with all R blocks of its own segment, ascending (as
 *   pbs_block_mask writes them), takes these R blocks from the token-order copy instead: the blocks before the
 *   diagonal in full, the diagonal block under the causal test, none after it.  These are the same visible keys,
 *   so O' and lse are the same up to the rounding order of the sums; every other list is processed as listed.
 */
pbs_status pbs_attn_fwd(const pbs_problem *p, const void *Qp, const void *Kp, const void *Vt,
                        const int32_t *qidx, const int32_t *kidx, const int32_t *row_cnt, const int32_t *col_idx,
                        void *Op, float *lse, void *ws, size_t ws_bytes, void *stream);

/*
 * Algorithm 1's last step (Theorem 1): O[qidx[slot]] = Op[slot].  qidx NULL (P_sigma = I, the paper's main
 * setting) makes this a plain copy, or nothing at all when O == Op.  Op, O [batch,h_q,n,d]; O must not
 * partially overlap Op.
 */
pbs_status pbs_unpermute(const pbs_problem *p, const void *Op, const int32_t *qidx, void *O, void *stream);

/*
 * Coverage tooling for the block-selection objective of Section "The Problem of Information Fragmentation" (the
 * attention mass, softmax over every visible key, that falls into the selected blocks); not a step of Algorithm 1.
 * pbs_admitted_lists writes the lists that name every key block the extended causal mask C admits (appendix "Block
 * Selection in PBS-Attn"): row_cnt[b,h,i] = (g(i)+1)*R capped at T inside full segment g(i), i+1 past the last full
 * segment; col_idx[b,h,i,0..row_cnt) = 0, 1, ...  (shapes as for pbs_block_mask; the rest of col_idx is untouched).
 * pbs_mass_covered combines the log-sum-exp outputs of two pbs_attn_fwd calls, one over a selection and one over the
 * admitted lists: covered[b,h,slot] = exp(lse_listed - lse_admitted), 0 where lse_listed is -inf.  All three
 * [batch,h_q,n] float32; covered may alias either input.
 * Errors: PBS_ERR_NULL, the statuses of pbs_validate, PBS_ERR_HIP.
 */
pbs_status pbs_admitted_lists(const pbs_problem *p, int32_t *row_cnt, int32_t *col_idx, void *stream);
pbs_status pbs_mass_covered(const pbs_problem *p, const float *lse_listed, const float *lse_admitted, float *covered,
                            void *stream);

/*
 * Measurement aids, not steps of Algorithm 1.
 * pbs_mfma_rate_probe launches a kernel that does nothing but bf16 matrix instructions (four waves per SIMD on 256
 * compute units, operands in registers, no other instruction in the loop) for `iters` rounds of 32 instructions, with
 * all-zero operands (random_operands = 0) or pseudo-random ones.  The caller times the launch on `stream`; *flop (host
 * memory) receives the number of floating-point operations it performs.  The instruction rate per clock is the same
 * in both cases; the clock the chip grants under matrix load depends on the operand bits, so the rate with random
 * operands is the matrix rate a kernel working on real data can approach.
 *   sink: device memory, sink_floats >= 262144 float32, overwritten; afterwards sink[0] = shader clock in MHz that one
 *   wave of the launch saw, sink[1] = that wave's clocks per matrix instruction (four waves share a SIMD: 4 x 32 in a
 *   long run).  iters in [1, 2^22].
 * pbs_shader_clock_meter launches one wave that compares the shader-clock counter with the constant 100 MHz counter
 * for about `micros` microseconds (1 .. 2 000 000) and writes out[0] = shader clock in MHz, out[1] = microseconds
 * watched (device memory, 2 floats).  Launched on a second stream beside another kernel it reports that kernel's clock.
 * Errors: PBS_ERR_NULL, PBS_ERR_SHAPE (a size or count out of range), PBS_ERR_HIP.
 */
pbs_status pbs_mfma_rate_probe(int random_operands, int iters, float *sink, size_t sink_floats, double *flop,
                               void *stream);
pbs_status pbs_shader_clock_meter(float *out, int micros, void *stream);

/*
 * ---------------------------------------------------------------------------------------------------------------
 * Around the prefill path: rotary positions in front of it, the paged key/value cache behind it, attention of new
 * tokens over that cache, and causal attention over packed prompts that are too short for block selection to pay.
 *
 * These calls see tensors as tokens x heads x features: element (t, h, e) of a tensor lies at t * strides.token +
 * h * strides.head + e, in elements; features are consecutive.  [tokens, heads, d] memory has strides {heads * d, d}, the
 * [1, heads, n, d] memory of the calls above {d, n * d}, and a slice of a fused projection its own.  Base addresses are
 * 16-byte aligned, strides are not negative, below 2^31 and whole multiples of 16 bytes; rows of an output do not overlap (all
 * PBS_ERR_SHAPE otherwise).  d is 64 or 128.  A count of zero tokens or sequences is a call that does nothing.  A launch has
 * fewer than 2^32 threads: a call that needs more of a kernel is PBS_ERR_UNSUPPORTED (pbs_rope from 2^24 workgroups of one to
 * eight tokens on, the cache from 2^35 / d rows, pbs_decode_attn from 2^26 rows of queries, 2^24 with a prefix or many pieces).
 * The other conventions above hold: host-validated, nothing allocated, no synchronisation, deterministic.
 */
typedef struct { int64_t token, head; } pbs_strides;

/*
 * Rotary positions.  Every head's first `rot` features are taken as rot / 2 pairs, pair e turned by the angle
 * position * freq[e] and multiplied by `magnitude`; the features behind them are copied:
 *     first'  = magnitude * (first * cos - second * sin),      second' = magnitude * (first * sin + second * cos).
 *   layout   PBS_ROPE_HALF: pair e is features (e, e + rot / 2); PBS_ROPE_INTERLEAVED: features (2e, 2e + 1).
 *   rot      a multiple of 16, at most d.
 *   flags    PBS_ROPE_TRANSPOSE: sin changes its sign: the gradient of the turned features with respect to the given
 *            ones, applied to Q and K (with magnitude 1 also the inverse).
 *   freq     [rot / 2] float64, device memory: radians per position, as pbs_rope_frequencies forms them.
 *   positions [tokens] int32, device memory, any sign; the same for all heads.
 *   Q, K     [tokens, h_q, d], [tokens, h_kv, d] of dtype PBS_BF16 or PBS_F32; h_q or h_kv (not both) may be 0, its
 *            pointers are then ignored.  Qout and Kout may be Q and K themselves with the same strides; other overlaps are
 *            not allowed.
 * The angle is formed and reduced to one turn in 64 bits; cos, sin and the products are fp32, rounded once at the end.
 * Errors: PBS_ERR_NULL, PBS_ERR_SHAPE, PBS_ERR_UNSUPPORTED (dtype, d, rot, layout, h_q + h_kv > 8192, more than 2^31 - 1
 * rows), PBS_ERR_HIP.
 */
enum { PBS_ROPE_HALF = 0, PBS_ROPE_INTERLEAVED = 1 };
enum { PBS_ROPE_TRANSPOSE = 1u };
typedef struct {
    int32_t tokens, h_q, h_kv, d, rot;
    int32_t layout;   /* PBS_ROPE_HALF or PBS_ROPE_INTERLEAVED */
    int32_t dtype;    /* of Q, K, Qout, Kout */
    float magnitude;  /* 0 means 1 */
    uint32_t flags;   /* PBS_ROPE_TRANSPOSE */
    pbs_strides q, k, q_out, k_out;
} pbs_rope_problem;
pbs_status pbs_rope(const pbs_rope_problem *p, const double *freq, const int32_t *positions, const void *Q,
                    const void *K, void *Qout, void *Kout, void *stream);

/*
 * The frequencies of the rotary pairs, f_e = base^(-2e / rot), and how they are scaled for contexts longer than the
 * `original` one.  Runs on the host; freq [rot / 2] and magnitude are HOST memory.
 *   PBS_ROPE_PLAIN   f_e.
 *   PBS_ROPE_LINEAR  f_e / factor (position interpolation).
 *   PBS_ROPE_BANDS   by the turns w_e = original * f_e / (2 pi) that a pair makes over the original context: keep =
 *                    clamp((w_e - low) / (high - low), 0, 1), f_e * (keep + (1 - keep) / factor).
 *   PBS_ROPE_RAMP    by the pair's index: i(w) = rot * ln(original / (2 pi w)) / (2 ln base), squeeze = clamp((e - a) /
 *                    max(b - a, 0.001), 0, 1) with a = max(floor(i(high)), 0), b = min(ceil(i(low)), rot - 1),
 *                    f_e * (1 - squeeze + squeeze / factor), and magnitude 0.1 ln(factor) + 1 (arXiv 2309.00071).
 * *magnitude receives 1 for the other three.  Errors: PBS_ERR_NULL; PBS_ERR_SHAPE unless rot is even and positive, base > 1,
 * factor >= 1, original >= 1 and 0 < low < high (each looked at where it is used); PBS_ERR_UNSUPPORTED for an unknown scaling.
 */
enum { PBS_ROPE_PLAIN = 0, PBS_ROPE_LINEAR = 1, PBS_ROPE_BANDS = 2, PBS_ROPE_RAMP = 3 };
pbs_status pbs_rope_frequencies(int scaling, int32_t rot, double base, double factor, double original, double low,
                                double high, double *freq, double *magnitude);

/*
 * A paged key/value cache.  Slot s = page number * page + place in the page holds one token's keys and values of every kv
 * head: row (h, place) of page K[page number], of `d` features.  What a row holds, for K and V alike:
 *   PBS_BF16   the features themselves; k_scale and v_scale are NULL.
 *   PBS_E4M3, PBS_I8   a factor f = max(|largest feature| / M, 2^-126) in fp32, M = 448 and 127, and every feature divided by f
 *              and rounded to the nearest value of the type, ties to even; the row stands for the products with f.  A
 *              row with an infinite or NaN feature holds the factor NaN and zeros: it reads back as NaN throughout.
 * K, V: device memory, 16-byte aligned, caller-owned like everything else.
 */
typedef struct {
    int32_t pages;     /* >= 1; pages * page <= 2^31 - 1 */
    int32_t page;      /* slots to a page: 16, 32, 64, ... 1024 */
    int32_t h_kv, d;
    int32_t dtype;     /* PBS_BF16, PBS_E4M3 or PBS_I8 */
    void *K, *V;       /* [pages, h_kv, page, d] */
    float *k_scale, *v_scale; /* [pages, h_kv, page] */
} pbs_cache;

/*
 * Writes the rows of `tokens` tokens into the cache: K, V [tokens, h_kv, d] of `dtype` (PBS_BF16 or PBS_F32) with the given
 * strides, slots [tokens] int32 in device memory.  A slot outside [0, pages * page) is passed over (the padding of a
 * batch).  The slots of one call have to differ from each other; two tokens with the same slot leave an undefined row there.
 * Every row that no slot names stays as it was.
 * pbs_cache_read is the way back: row t of K, V [tokens, h_kv, d] of `dtype` becomes what slot slots[t] stands for
 * (the held value times its factor in fp32, rounded to dtype), zeros for a slot outside the cache.  K or V may be NULL
 * (then it is not read back); slots may repeat.
 * Errors: PBS_ERR_NULL, PBS_ERR_SHAPE, PBS_ERR_UNSUPPORTED (dtype, d, page, h_kv > 65535, more than 2^31 - 1 slots,
 * 2^35 / d rows or more), PBS_ERR_HIP.
 */
pbs_status pbs_cache_write(const pbs_cache *c, int32_t dtype, int32_t tokens, const void *K, const pbs_strides *k,
                           const void *V, const pbs_strides *v, const int32_t *slots, void *stream);
pbs_status pbs_cache_read(const pbs_cache *c, int32_t dtype, int32_t tokens, const int32_t *slots, void *K,
                          const pbs_strides *k, void *V, const pbs_strides *v, void *stream);

/*
 * Attention of each sequence's newest q_len tokens over its cached keys, a prefix that all sequences share in front of
 * them: query t of sequence i sees all prefix_len prefix keys and its own keys 0 .. lens[i] - q_len + t (its own keys
 * include the new tokens, written before this call).  O = softmax(scale * Q K^T) V over these; a query that sees none gets a
 * zero row and lse = -inf, as does one whose logits are all -inf.
 *   Q, O     token i * q_len + t; dtype bf16 whatever the cache holds; h_q % c->h_kv == 0.  O may be Q itself with
 *            the same strides (PBS_ERR_SHAPE otherwise); other overlaps are not allowed.
 *   page_table [n_seq, max_pages] int32: the pages of a sequence's own keys in order; entries behind its length are
 *            not looked at.  A listed page outside [0, pages) counts as keys that nobody sees.
 *   lens     [n_seq] int32, device memory: own keys; negative counts as 0, more than min(max_len, max_pages * page) as that.
 *   max_len  an upper bound of lens that the host knows; how the work is cut follows lens themselves, but a small bound
 *            needs fewer workgroups and no workspace (without a prefix: up to 128, with many sequences up to 512).
 *   prefix_pages [ceil(prefix_len / page)] int32, device memory; NULL when prefix_len is 0.  The prefix is read for 16 to
 *            128 rows (query, head of its group) of the whole batch at a time, not once per sequence.
 *   lse      [n_seq * q_len, h_q] float32 or NULL: log-sum-exp of the logits that each query sees.
 *   ws       pbs_decode_workspace_bytes(p, c) bytes, 256-byte aligned (0: may be NULL); need not be initialised, means
 *            nothing afterwards.  Calls that may overlap in time need one each.  Behind a prefix it holds d + 2 floats for every
 *            row of Q and part of the prefix (1024 keys at most where it is read for 128 rows at a time: 256 rows of 32 heads of 128
 *            behind 131072 keys take 545 MB), and, there and in 8 bits, the prefix in bf16; without one d + 2 floats for the
 *            rows, 32 at most, of every (sequence, kv head) and of 2048 pieces (4096 sequences of 8 kv heads 73 MB).
 * Probabilities, with a value row's factor in them, enter the second product as two terms in bf16 (2^-16 of each is lost at most), against
 * a prefix that is read for 128 rows at a time as one (2^-8 at most); everything else is fp32.
 * Errors: PBS_ERR_NULL, PBS_ERR_SHAPE (max_len or prefix_len negative, misaligned, a scale that is negative or not
 * finite), PBS_ERR_UNSUPPORTED (q_len > 16, n_seq > 65535, n_seq * q_len * h_q or n_seq * max_pages > 2^31 - 1,
 * max_len > 2^27, prefix_len > 2^25, a grid that is too large, dtype), PBS_ERR_WORKSPACE, PBS_ERR_HIP.
 */
typedef struct {
    int32_t n_seq, q_len, h_q;
    int32_t max_pages, max_len, prefix_len;
    int32_t dtype;    /* of Q and O: PBS_BF16 */
    float scale;      /* 0 means 1/sqrt(d) */
    pbs_strides q, o;
} pbs_decode_problem;
size_t pbs_decode_workspace_bytes(const pbs_decode_problem *p, const pbs_cache *c);
pbs_status pbs_decode_attn(const pbs_decode_problem *p, const pbs_cache *c, const void *Q, const int32_t *page_table,
                           const int32_t *lens, const int32_t *prefix_pages, void *O, float *lse, void *ws,
                           size_t ws_bytes, void *stream);

/*
 * Attention over prompts packed one behind the other.  Sequence i has the query rows cu_q[i] .. cu_q[i+1] - 1 and the key
 * rows cu_k[i] .. cu_k[i+1] - 1 (cu_q, cu_k [n_seq + 1] int32, device memory, ascending; a place outside [0, total_q] or
 * [0, total_k] is taken as the nearest inside, a length below zero as zero).  With PBS_PROMPT_CAUSAL query t of a sequence sees
 * key j iff j <= t + (number of keys) - (number of queries): the newest query sees everything, as when a chunk of a
 * prompt follows keys that are there already; without it every query sees every key of its sequence.  A query that sees no
 * key, or whose logits are all -inf, gets a zero row and lse = -inf.  Rows of O and lse that belong to no sequence stay as they were.
 *   Q, O [total_q, h_q, d], K, V [total_k, h_kv, d], bf16; h_q % h_kv == 0, h_q / h_kv <= 128; lse [total_q, h_q] float32 or NULL.
 *   O may not overlap Q, K or V (PBS_ERR_SHAPE where it starts at one of them).
 * Probabilities enter the second product rounded to bf16 (off by 2^-8 of each at most), everything else is fp32.
 * Errors: PBS_ERR_NULL, PBS_ERR_SHAPE, PBS_ERR_UNSUPPORTED (dtype, d, h_q / h_kv > 128, rows beyond 2^31 - 1, a grid that is
 * too large, K or V of one head spanning 2 GiB or more), PBS_ERR_HIP.
 */
enum { PBS_PROMPT_CAUSAL = 1u };
typedef struct {
    int32_t n_seq, total_q, total_k;
    int32_t h_q, h_kv, d;
    int32_t dtype;    /* PBS_BF16 */
    float scale;      /* 0 means 1/sqrt(d) */
    uint32_t flags;   /* PBS_PROMPT_CAUSAL */
    pbs_strides q, k, v, o;
} pbs_prompt_problem;
pbs_status pbs_prompt_attn(const pbs_prompt_problem *p, const void *Q, const void *K, const void *V, const int32_t *cu_q,
                           const int32_t *cu_k, void *O, float *lse, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PBS_H */
