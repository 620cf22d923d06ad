/* disc.h - C ABI of the B200 (sm_100a) DISC + PPV constrained-decoding hot path.
 *
 * The library implements the per-step work of the paper "Efficient and Asymptotically Unbiased
 * Constrained Decoding for Large Language Models" (DISC, Algorithm 1; PPV, Algorithm 2):
 *
 *   disc_build_set   Algorithm 2, line 1 ("Prepare") and Section 3.2 "Array Preparation": sort the
 *                    members of S lexicographically by token id and keep the array on the GPU.
 *   disc_mask        Algorithm 2, lines 3-7 with M = |V|: the mask of the valid set A_{a,S}
 *                    (Section 2.1) of a prefix a.
 *   disc_verify      Algorithm 2, lines 4-6 as stated: M candidate tokens per prefix verified by
 *                    binary search in the sorted array (top-M mode).
 *   disc_topm        Algorithm 2, line 3: the M most probable tokens of every row.
 *   disc_step_topm   Algorithm 1, lines 5-8 with the mask of Algorithm 2 as the paper runs it: the
 *                    top-M tokens are verified against the sorted array and the token is drawn
 *                    among the verified ones.
 *   disc_step        Algorithm 1, lines 5-8 for a batch of partial sequences: mask, sample from
 *                    P.mask/|P.mask|_1, append, multiply the importance score by |P.mask|_1.
 *   disc_project_step  the same step with line 5's P = L(a, T) folded in: the model's last projection
 *                    (hidden vectors times the vocabulary matrix) runs on the tensor cores and
 *                    only the pieces of the logits the step looks at ever reach memory.
 *   disc_resample    Algorithm 1, line 22: among K finished candidates pick one with probability
 *                    x_k / sum_j x_j.
 *   disc_accept      Algorithm 1, line 16: accept a candidate when x > eps ~ U[0,1].
 *   disc_accept_resample  Algorithm 1, lines 11-22: K ordered accept tests, then the K-way draw
 *                    over K fresh candidates.
 *
 * and what the language model around it runs for B queries with K candidates each (line 5's
 * P = L(a, T) with a model of attention layers):
 *
 *   disc_attend_prompt   attention over whole prompts, packed
 *   disc_norm_rope, disc_norm_rope_grad   head norms and rotation of queries and keys, and their gradient
 *   disc_cache_*         a key-value cache in pages that the candidates of a query share: fork,
 *                    extend, write, read, free, compact; its vectors as they are or held in 8 bits
 *   disc_norm_rope_write  norm, rotation and the way into the cache in one launch
 *   disc_attend_plan, disc_attend_cached   attention of one new token per candidate over that cache
 *   disc_logprobs, disc_logprobs_grad   log-probabilities of given tokens, entropy, the most probable
 *                    alternatives, and the gradient for training on them
 *
 * Conventions
 *   - Every function returns 0 (DISC_OK) or a negative DISC_ERR_* code.  Return codes cover
 *     argument validation and CUDA launch/allocation errors only; problems of a single row are
 *     reported in that row's status byte and never fail the call.
 *   - "host" pointers are ordinary CPU memory, "device" pointers are memory of the current CUDA
 *     device, owned by the caller.  `stream` is a cudaStream_t (NULL = the default stream).
 *     A handle belongs to the device that was current when it was built; calls that take a
 *     handle return DISC_ERR_ARG when another device is current.
 *   - Except for disc_build_set / disc_free_set / disc_set_info / disc_set_rows, calls only enqueue
 *     kernels on `stream`: they allocate nothing, do not synchronise the host, and finish in
 *     stream order.
 *   - The importance score x of Algorithm 1 is kept as its logarithm `logw` in fp32 (x starts at 1,
 *     logw at 0; each step adds log |P.mask|_1).
 *   - The set must be prefix-free (all members of one length, or every member closed by an
 *     end-of-sequence token that is an ordinary token): "a in S" (Algorithm 1, line 4) is then
 *     "a's node has no child".
 *   - Mask layout: W = ceil(V/32) uint32 words per row; token v is bit (v & 31) of word (v >> 5);
 *     bits at positions >= V are zero.
 *   - Random numbers: Philox4x32-10, key = (seed low 32 bits, seed high 32 bits).  The uniform of
 *     output word r is u = ((r >> 9) + 0.5) * 2^-23 (u and 1-u exact in fp32).  Counters:
 *       group noise  (((G>>10)<<8) | (G&255), step, row, 0), word (G>>8)&3   per token group G
 *       in-group     (G, step, row, 3), word 0
 *       resample     (query, 0, 0, 1), word 0
 *       accept       (query, k, 0, 2), word 0
 *     where `row` / `query` is row_base / query_base plus the index inside the call.  Each is one
 *     32-bit counter word: row_base + n and query_base + B must not exceed 2^32
 *     (DISC_ERR_UNSUPPORTED otherwise).
 *   - Sampling draws exactly from P.mask/|P.mask|_1 in two stages.  Tokens are taken in groups of
 *     8 consecutive ids (G = v >> 3).  Stage 1 is Gumbel-max over groups: the group maximising
 *     log(sum of e^{z_v/T} over its allowed tokens) - log(-log u_G) wins (the lowest G on an exact
 *     tie); it is therefore chosen with probability proportional to its allowed mass.  Stage 2
 *     picks, inside the winner, the smallest allowed token whose inclusive cumulative weight
 *     exceeds u' * mass (tokens in ascending id).
 */
#ifndef DISC_H_
#define DISC_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DISC_OK 0
#define DISC_ERR_ARG (-1)         /* null, negative, out-of-range or misaligned argument          */
#define DISC_ERR_EMPTY (-2)       /* empty set or empty member                                    */
#define DISC_ERR_TOKEN (-3)       /* token id outside [0, vocab_size)                             */
#define DISC_ERR_PREFIX (-4)      /* a member is a proper prefix of another member                */
#define DISC_ERR_OOM (-5)         /* device or host allocation failed                             */
#define DISC_ERR_CUDA (-6)        /* a CUDA call failed; see disc_last_cuda_error()               */
#define DISC_ERR_UNSUPPORTED (-7) /* size or dtype outside what the kernels support               */

/* per-row status bits */
#define DISC_ROW_DEAD 1     /* prefix / node is not a prefix of any member                        */
#define DISC_ROW_NOMASS 2   /* allowed probability mass is zero or not finite                     */
#define DISC_ROW_NONFINITE 4 /* NaN or +Inf among the row's logits (or NaN among the weights)     */
#define DISC_ROW_DONE 8     /* row was already complete: nothing read, state untouched            */
#define DISC_ROW_FAULT 16   /* reserved for kernels that wait inside the device; no present kernel sets it
                               (disc_project_step reports a wait that ran out through
                               disc_project_error instead)                                        */
#define DISC_ROW_NOPAGE 32  /* the cache has no room for the row's new tokens; the row is unchanged   */

typedef struct disc_set disc_set_t; /* opaque; owns its device memory */

typedef enum { DISC_F32 = 0, DISC_BF16 = 1, DISC_F16 = 2 /* attention and cache only */ } disc_dtype_t;

#define DISC_MAX_DEPTH 64

typedef struct {
    int64_t n_members;       /* N: members after de-duplication                                  */
    int64_t n_entries;       /* E: int32 entries of the sorted table                             */
    int64_t n_nodes;         /* distinct non-empty prefixes of members (index nodes)             */
    int32_t vocab_size;      /* V                                                                */
    int32_t mask_words;      /* W = ceil(V/32)                                                   */
    int32_t l_max;           /* longest member                                                   */
    int32_t n_heavy;         /* nodes with more than 1024 children (their masks are prebuilt)    */
    int64_t device_bytes;    /* device memory held by the handle                                 */
    double build_seconds;    /* wall time of disc_build_set                                      */
    int64_t level_nodes[DISC_MAX_DEPTH]; /* distinct prefixes of length d+1, d = 0..l_max-1      */
} disc_set_info_t;

/* Build the device-resident constraint array (Algorithm 2, line 1; Section 3.2 "Array
 * Preparation").
 *   tokens       host, int32[row_offsets[n_rows]]: the members back to back, in any order
 *   row_offsets  host, int64[n_rows+1]: member r is tokens[row_offsets[r] .. row_offsets[r+1])
 *   vocab_size   V; every token must lie in [0, V)
 *   flags        must be 0
 *   stream       stream the build kernels run on; the call synchronises it before returning
 *   out          receives the handle (NULL on error)
 * The inputs are copied.  Members are sorted lexicographically by token id (a shorter sequence
 * before its extensions), duplicates are collapsed.  Besides the sorted table the handle holds an
 * index with one node per distinct non-empty prefix, level by level, from which the valid set of
 * any prefix is read as a contiguous list.
 * Errors: DISC_ERR_ARG, DISC_ERR_EMPTY (no member / an empty member), DISC_ERR_TOKEN,
 * DISC_ERR_PREFIX, DISC_ERR_UNSUPPORTED (n_rows >= 2^31, entries >= 2^32, member longer than
 * DISC_MAX_DEPTH, V > 4,000,000), DISC_ERR_OOM, DISC_ERR_CUDA. */
int disc_build_set(const int32_t* tokens, const int64_t* row_offsets, int64_t n_rows,
                   int32_t vocab_size, uint32_t flags, void* stream, disc_set_t** out);

/* The same build for sets in which a member may be a proper prefix of another member (Section 2.1
 * lets the model stop at a member by emitting an end-of-keyword token there).  Every member is
 * closed by eok_token (on a host copy; the caller's arrays are not changed), which makes the set
 * prefix-free, and disc_build_set follows.  Afterwards the valid set of a prefix that is itself a
 * member contains eok_token next to the tokens that extend it, and a candidate is complete once
 * it has produced eok_token; sequences returned by disc_step / disc_resample end with it.
 *   eok_token   in [0, vocab_size); must not occur inside any member (DISC_ERR_TOKEN otherwise)
 * The longest member may have DISC_MAX_DEPTH - 1 tokens.  Other arguments and errors as for
 * disc_build_set (DISC_ERR_PREFIX cannot occur). */
int disc_build_set_eok(const int32_t* tokens, const int64_t* row_offsets, int64_t n_rows,
                       int32_t vocab_size, int32_t eok_token, void* stream, disc_set_t** out);

/* Release the handle and its device memory.  NULL is allowed. */
void disc_free_set(disc_set_t* s);

/* Sizes of the built set.  `info` is host memory. */
int disc_set_info(const disc_set_t* s, disc_set_info_t* info);

/* Copy the sorted, de-duplicated table back (the array X of Algorithm 2, without padding).
 *   tokens_out       host, int32[n_entries]
 *   row_offsets_out  host, int64[n_members+1]
 * Synchronises the device. */
int disc_set_rows(const disc_set_t* s, int32_t* tokens_out, int64_t* row_offsets_out);

/* Start n candidates at the empty sequence (Algorithm 1, line 3: a = [], x = 1).
 * All arrays are device memory with n entries: node = root, [lo, hi) = [0, N), depth = 0,
 * logw = 0, done = 0. */
int disc_state_init(const disc_set_t* s, int64_t n, int32_t* node, int32_t* lo, int32_t* hi,
                    int32_t* depth, float* logw, uint8_t* done, void* stream);

/* Valid-set masks of n prefixes (Algorithm 2, lines 3-7 in the M = |V| limit; Section 2.1).
 *   prefix      device, int32[n][prefix_ld]; row i holds prefix_len[i] tokens
 *   prefix_len  device, int32[n], 0 <= prefix_len[i] <= prefix_ld
 *   mask_out    device, uint32[n][W] (nullable): bit v set iff prefix+[v] is a prefix of a member
 *   lo_out, hi_out  device, int32[n] (nullable): the members having the prefix are rows [lo, hi)
 *               of the sorted table
 *   node_out    device, int32[n] (nullable): index node of the prefix (the cursor disc_step uses)
 *   status_out  device, uint8[n]: 0, or DISC_ROW_DEAD when the prefix is a prefix of no member
 *               (then the mask is zero and lo = hi = node = -1)
 * A complete member has an empty mask and a range of one row.
 * With mask_out given, the call keeps a row counter in the set handle: two such calls on the
 * same handle must not run on the device at the same time (calls issued to one stream never do;
 * calls on different streams need an event between them, or a handle each).  n must be below
 * 2^31 - 2^20 (DISC_ERR_UNSUPPORTED otherwise). */
int disc_mask(const disc_set_t* s, const int32_t* prefix, int32_t prefix_ld,
              const int32_t* prefix_len, int64_t n, uint32_t* mask_out, int32_t* lo_out,
              int32_t* hi_out, int32_t* node_out, uint8_t* status_out, void* stream);

/* disc_mask with the writer's row counter in a fixed word block inside the loaded module (a
 * file-scope device array of 256 bytes per device) instead of device memory obtained from the
 * allocator.  The paper has no counterpart of this entry point; it exists for callers that cannot
 * let a library allocate device memory on their behalf: a serving process that sizes its own pool
 * to all of the memory left at start-up has no room to give later, and an allocation made behind
 * its back can fail or push it over its budget.  This call performs no allocation and frees
 * nothing, on the device or through the CUDA allocator.
 * Arguments, outputs and errors are those of disc_mask.  In addition:
 *   - n must not exceed DISC_MASK_STATIC_MAX_ROWS; a larger n is refused with DISC_ERR_UNSUPPORTED
 *     before anything is launched;
 *   - the first call on a device looks up the address of the word block (with that device
 *     current) and keeps it; make that first call outside any stream capture;
 *   - the block is shared by every call on that device, whatever the handle or stream: two calls
 *     must not run on the device at the same time (calls on one stream never do).  Nothing has to be
 *     cleared between calls: the first kernel of each call resets the counter, and what an earlier
 *     call left there is never read. */
#define DISC_MASK_STATIC_MAX_ROWS 1073741824 /* 2^30 prefixes per call */
int disc_mask_static(const disc_set_t* s, const int32_t* prefix, int32_t prefix_ld,
                     const int32_t* prefix_len, int64_t n, uint32_t* mask_out, int32_t* lo_out,
                     int32_t* hi_out, int32_t* node_out, uint8_t* status_out, void* stream);

/* Algorithm 2 as stated (lines 4-6; Section 3.2 "Parallel Verification"): for each of n partial
 * sequences a and each of its M candidate tokens t_m, find by binary search in the sorted member
 * array X the smallest row that is not lexicographically smaller than V_m = a + [t_m]; t_m is
 * valid iff V_m is a prefix of that row.  Only the sorted table is read, not the prefix index.
 *   prefix, prefix_ld, prefix_len   as for disc_mask (0 <= prefix_len[i] <= prefix_ld, at most
 *               DISC_MAX_DEPTH; a prefix outside that gets the empty range [0, 0))
 *   cand        device, int32[n][M]: the candidates (for instance the top-M tokens of P); ids
 *               outside [0, V) are invalid
 *   valid_out   device, uint8[n][M]: mask_V of Algorithm 2, line 5
 *   row_out     device, int32[n][M] (nullable): the row index the search lands on (N when every
 *               row is smaller)
 *   mask_out    device, uint32[n][W] (nullable): line 6, bit t_m set iff t_m is valid, all other
 *               bits zero; with every token among the candidates this is disc_mask's mask
 *   lo_out, hi_out  device, int32[n] (required): the rows having a as a prefix are [lo, hi) (empty
 *               range with lo = hi = insertion point when there is none)
 * M = 0 computes the ranges only.  Errors: DISC_ERR_ARG; DISC_ERR_UNSUPPORTED when n*M >= 2^38. */
int disc_verify(const disc_set_t* s, const int32_t* prefix, int32_t prefix_ld, const int32_t* prefix_len,
                int64_t n, const int32_t* cand, int32_t M, uint8_t* valid_out, int32_t* row_out,
                uint32_t* mask_out, int32_t* lo_out, int32_t* hi_out, void* stream);

/* One decoding step for n candidates (Algorithm 1, lines 5-8; score closed form in Appendix A).
 *   logits   device, n rows of V values of type `dtype`, row i at element offset i*ld.  The fast
 *            path needs the base 16-byte aligned and ld*sizeof(value) a multiple of 16; other
 *            layouts take a slower scalar path.  Pinned (page-locked, device-accessible) host
 *            memory is accepted as well: the kernel then reads it in place over PCIe, and rows
 *            that are already complete are not read at all.
 *   inv_temperature  1/T (Algorithm 1's T), finite and > 0
 *   seed, step, row_base  random-number coordinates (see top of file); `step` must differ between
 *            the steps of one decode
 *   node, lo, hi, depth, logw, done   device, in/out state, n entries each
 *   token_out   device, int32[n]: sampled token, -1 for rows that did nothing
 *   seq_tokens  device, int32[n][seq_ld] (nullable): the token is also stored at
 *            seq_tokens[i][depth[i]] (depth before the step) when depth[i] < seq_ld
 *   logq_out    device, float[n] (nullable): log-probability of the token under the masked,
 *            renormalised distribution
 *   logp_out    device, float[n] (nullable): its log-probability under the unmasked distribution
 *   mask_out    device, uint32[n][W] (nullable): the valid-set mask used by each live row
 *   status_out  device, uint8[n]
 * Per live row: z_v = logit_v / T; lse_all = log sum_v e^{z_v}; lse_ok = the same over the valid
 * set; logw += lse_ok - lse_all; token drawn from the valid set (two-stage rule at the top of this
 * file); the state moves to the extended prefix; done is set when the extended prefix is a member.
 * Rows with done != 0 are skipped (status DISC_ROW_DONE, token -1, no logits read).  A row whose
 * valid mass is zero keeps going with the lowest valid token (status DISC_ROW_NOMASS,
 * logw = -inf); NaN/+Inf logits give status DISC_ROW_NONFINITE, a NaN/Inf logw and some valid
 * token (which one is unspecified). */
int disc_step(const disc_set_t* s, const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n,
              float inv_temperature, uint64_t seed, uint32_t step, int64_t row_base,
              int32_t* node, int32_t* lo, int32_t* hi, int32_t* depth, float* logw, uint8_t* done,
              int32_t* token_out, int32_t* seq_tokens, int32_t seq_ld, float* logq_out,
              float* logp_out, uint32_t* mask_out, uint8_t* status_out, void* stream);

/* Algorithm 2, line 3: the M tokens of largest logit of each of n rows (the M most probable ones).
 * Equal logits (-0 and +0 are equal) are ordered by token id, the lower id first; NaN logits come
 * last.  The selection is exact for every input.
 *   logits, dtype, ld   as for disc_step (device memory; rows of vocab_size values)
 *   done        device, uint8[n] (nullable): rows with done != 0 are skipped (candidates -1)
 *   cand_out    device, int32[n][M]: the selected token ids in ascending order, -1 padded when
 *               M > vocab_size
 *   lse_out     device, float[n][2] (nullable): the pair (m, s) with
 *               sum_v 2^(logit_v * log2(e) * inv_temperature) = 2^m * s, a by-product of the passes
 *               over the row (inv_temperature is used for this output only)
 * Errors: DISC_ERR_ARG, DISC_ERR_UNSUPPORTED (dtype; n >= 2^31). */
int disc_topm(const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n, int32_t vocab_size, int32_t M,
              float inv_temperature, const uint8_t* done, int32_t* cand_out, float* lse_out, void* stream);

/* One decoding step in the paper's top-M mode (Algorithm 1, lines 5-8, with mask = PPV_S(P, a) computed
 * as Algorithm 2 states it: line 3 selects the M most probable tokens, lines 4-5 verify each
 * a + [t_m] by binary search in the sorted array, line 6 is the mask of the verified ones).  The
 * token is drawn among the verified candidates by disc_step's two-stage rule, the importance
 * log-weight grows by the log of their probability mass.  With M = |V| the result is disc_step's.
 * A row none of whose candidates is valid has reached a dead end: it would fail Algorithm 1's test
 * "a in S" (line 15), so it ends here with status DISC_ROW_DEAD, token -1, done = 1 and
 * logw = -inf (the K-way draw then never picks it).
 *   M           1 <= M <= 1024
 *   seq_tokens  device, int32[n][seq_ld], required, seq_ld >= l_max: the tokens produced so far
 *               (the prefix a of every row, which the verification searches for); the new token
 *               is appended as in disc_step
 *   cand_out    device, int32[n][M]: receives the candidates (ascending id)
 *   scratch     device, disc_step_topm_scratch_bytes(n, M) bytes, 8-byte aligned, caller-owned
 *   other arguments as for disc_step (mask_out receives the mask of the verified candidates)
 * Four kernels are enqueued on `stream` (selection, prefix ranges and candidate verification, step). */
int64_t disc_step_topm_scratch_bytes(int64_t n, int32_t M);
int disc_step_topm(const disc_set_t* s, const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n, int32_t M,
                   float inv_temperature, uint64_t seed, uint32_t step, int64_t row_base, int32_t* node, int32_t* lo,
                   int32_t* hi, int32_t* depth, float* logw, uint8_t* done, int32_t* token_out, int32_t* seq_tokens,
                   int32_t seq_ld, float* logq_out, float* logp_out, uint32_t* mask_out, uint8_t* status_out,
                   int32_t* cand_out, void* scratch, int64_t scratch_bytes, void* stream);

/* One decoding step with the language model's last projection fused in (Algorithm 1, lines 5-8,
 * where line 5's next-token distribution is softmax(h W / T) of the model's final hidden vectors).
 *   logit[i][v] = bf16( sum_k hidden[i][k] * wt[v][k] )       (fp32 accumulation, rounded once to
 * bf16: the value a separate projection would have stored), then exactly disc_step on those logits.
 * The projection runs on the tensor cores; per row it keeps the sums the log-sum-exp over the
 * whole vocabulary needs, and writes logits only for the 256-wide vocabulary tiles that hold a
 * valid next token of the row (all tiles for a row at the empty prefix or at a node with more than
 * 1024 children), so that for the typical row deep in the prefix tree 512 bytes instead of 2V reach
 * memory.
 *   hidden      device, bf16[n][hidden_ld], d values used per row
 *   wt          device, bf16[V][wt_ld], d values used per row: the vocabulary projection, one
 *               vocabulary entry per row
 *   d           model width; a multiple of 8.  hidden, wt, logits_buf and scratch must be 16-byte
 *               aligned and the row pitches multiples of 16 bytes (DISC_ERR_ARG /
 *               DISC_ERR_UNSUPPORTED otherwise)
 *   inv_temperature, seed, step, row_base, state arrays, token_out, seq_tokens, seq_ld, logq_out,
 *   logp_out, status_out      as for disc_step
 *   logits_buf  device, bf16[n][logits_ld], logits_ld >= V: receives the logits pieces; with
 *               store_all != 0 every logit is written (the complete matrix a separate projection
 *               would have produced: for tests and diagnostics), otherwise what is not written
 *               keeps its old contents
 *   scratch     device, disc_project_scratch_bytes(s, n) bytes, caller-owned; its first word is an
 *               error flag the call clears and the kernel sets when one of its bounded waits ran
 *               out (read it with disc_project_error)
 * Rows with NaN or +-Inf logits get DISC_ROW_NONFINITE / DISC_ROW_NOMASS as in disc_step; their
 * log-weights are not finite but need not equal disc_step's bit for bit.
 * Three kernels are enqueued on `stream` (tile flags, projection, step); nothing is allocated. */
int64_t disc_project_scratch_bytes(const disc_set_t* s, int64_t n);
int disc_project_step(const disc_set_t* s, const void* hidden, int64_t hidden_ld, const void* wt, int64_t wt_ld,
                      int32_t d, int64_t n, float inv_temperature, uint64_t seed, uint32_t step, int64_t row_base,
                      int32_t* node, int32_t* lo, int32_t* hi, int32_t* depth, float* logw, uint8_t* done,
                      int32_t* token_out, int32_t* seq_tokens, int32_t seq_ld, float* logq_out, float* logp_out,
                      uint8_t* status_out, void* logits_buf, int64_t logits_ld, int32_t store_all, void* scratch,
                      int64_t scratch_bytes, void* stream);

/* Synchronises `stream` and returns DISC_ERR_CUDA when the projection kernel of an earlier
 * disc_project_step with this scratch buffer gave up on one of its waits (its results are then
 * invalid), DISC_OK otherwise. */
int disc_project_error(const void* scratch, void* stream);

/* K-way importance draw (Algorithm 1, line 22; Appendix A).
 *   logw        device, float[B][K]: log importance scores of the K candidates of each query
 *   idx_out     device, int32[B]: chosen candidate, P(k) = x_k / sum_j x_j
 *   logz_out    device, float[B] (nullable): log((1/K) sum_k x_k), an estimate of log P_L(S)
 *   seq_tokens  device, int32[B][K][seq_ld] (nullable) and tokens_out device int32[B][seq_ld]
 *               (nullable): when both are given the chosen candidate's tokens are copied out
 *   status_out  device, uint8[B]: DISC_ROW_NOMASS when no candidate has a finite positive weight
 *               (the pick is then uniform), DISC_ROW_NONFINITE when a weight is NaN (it counts as 0)
 * The pick is the smallest k whose inclusive prefix sum of weights exceeds u * total. */
int disc_resample(const float* logw, int32_t B, int32_t K, uint64_t seed, int64_t query_base,
                  int32_t* idx_out, float* logz_out, const int32_t* seq_tokens, int32_t seq_ld,
                  int32_t* tokens_out, uint8_t* status_out, void* stream);

/* Accept test over K finished candidates per query, in order (Algorithm 1, lines 12-21):
 *   first_out   device, int32[B]: smallest k with logw[b][k] > log(eps_{b,k}), eps uniform in
 *               (0,1); -1 when all K candidates are rejected (the caller then falls back to
 *               disc_resample on K fresh candidates). */
int disc_accept(const float* logw, int32_t B, int32_t K, uint64_t seed, int64_t query_base,
                int32_t* first_out, void* stream);

/* Algorithm 1, lines 11-22 for B queries with 2K finished candidates each: candidates 0..K-1 are
 * put to the accept test in order (line 16, as disc_accept); the first accepted one is returned;
 * when all K are rejected, one of the fresh candidates K..2K-1 is drawn with probability
 * x_k / sum_j x_j (line 22, as disc_resample over those K).  The output then follows
 * (1 - p_b^K) P_S + p_b^K Q_K (Appendix A), p_b = 1 - P_L(S).
 *   logw        device, float[B][2K]
 *   choice_out  device, int32[B]: the candidate returned, in [0, 2K)
 *   first_out   device, int32[B] (nullable): the accepted candidate, or -1 after K rejections
 *   logz_out    device, float[B] (nullable): log((1/K) sum x) over the fresh candidates
 *   seq_tokens  device, int32[B][2K][seq_ld] (nullable) with tokens_out int32[B][seq_ld] (nullable):
 *               the returned candidate's tokens are copied out
 *   status_out  device, uint8[B]: status of the K-way draw over the fresh candidates (see
 *               disc_resample); it matters only where first_out is -1
 * Random numbers: those of disc_accept and disc_resample for the same seed and query. */
int disc_accept_resample(const float* logw, int32_t B, int32_t K, uint64_t seed, int64_t query_base,
                         int32_t* choice_out, int32_t* first_out, float* logz_out,
                         const int32_t* seq_tokens, int32_t seq_ld, int32_t* tokens_out,
                         uint8_t* status_out, void* stream);

/* ---- log-probabilities ---------------------------------------------------------------------------
 * For each of n rows, with p = softmax(z / T) over the whole vocabulary:
 *   logits, dtype, ld   as for disc_step (any alignment of the rows; device memory)
 *   targets     device, int32[n] (nullable): the token to score; -1 = none (logp 0)
 *   top         0..64 alternatives per row
 *   logp_out    device, float[n] (required with targets): log p_target
 *   entropy_out device, float[n] (nullable): - sum_v p_v log p_v (nats)
 *   lse_out     device, float[n] (nullable): log sum_v e^{z_v/T}
 *   top_ids_out device, int32[n][top]: the most probable tokens in descending order; equal logits
 *               (-0 = +0) by the lower id first, NaN last; -1 beyond the vocabulary
 *   top_logp_out  device, float[n][top] (nullable): their log-probabilities (-inf beside a -1)
 *   status_out  device, uint8[n]: DISC_ROW_NOMASS for a row of -inf logits (lse and all
 *               log-probabilities -inf, entropy 0), DISC_ROW_NONFINITE for NaN or +inf among the logits
 *               (log-probabilities and entropy are then NaN or unspecified; the ids are not),
 *               DISC_ROW_DEAD for a target that is neither -1 nor in [0, vocab_size) (logp NaN)
 * Sums are held in fp32 relative to the row's maximum.
 * Errors: DISC_ERR_ARG, DISC_ERR_UNSUPPORTED (dtype; top > 64; n > 2^27). */
int disc_logprobs(const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n, int32_t vocab_size, float inv_temperature,
                  const int32_t* targets, int32_t top, float* logp_out, float* entropy_out, float* lse_out,
                  int32_t* top_ids_out, float* top_logp_out, uint8_t* status_out, void* stream);

/* The gradient of sum_i (d_logp[i] logp[i] + d_entropy[i] entropy[i]) with respect to the logits:
 *   grad[i][v] = (d_logp [v = target] - p_v (d_logp + d_entropy (log p_v + entropy))) / T
 *   lse, entropy   device, float[n]: what disc_logprobs returned for these logits (entropy nullable
 *               without d_entropy)
 *               (rows with |lse| >= 128, which fp32 holds too coarsely, have their sum formed anew; an lse
 *               that differs from it by more than 2^-21 of its size, a longer row's say, is taken as given)
 *   d_logp      device, float[n] (nullable; needs targets); rows without a target ignore it
 *   d_entropy   device, float[n] (nullable)
 *   grad_out    device, n rows of vocab_size values of type `dtype`, row i at element offset
 *               i*grad_ld; may be `logits` itself (with grad_ld = ld), otherwise must not overlap it
 * Rows of -inf logits get a zero gradient, rows with a non-finite lse a non-finite one. */
int disc_logprobs_grad(const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n, int32_t vocab_size, float inv_temperature,
                       const int32_t* targets, const float* lse, const float* entropy, const float* d_logp, const float* d_entropy,
                       void* grad_out, int64_t grad_ld, void* stream);

/* ---- attention over whole prompts ------------------------------------------------------------------
 * Packed sequences: sequence i has the queries cu_q[i] .. cu_q[i+1]-1 and the keys cu_k[i] ..
 * cu_k[i+1]-1 (lq and lk of them).  Query j of a sequence sees its keys 0 .. j + lk - lq with `causal`
 * (the last query sees all; a query that sees none gets out = 0, lse = -inf), all lk of them without.
 * Query head h reads key head h / (n_q_heads / n_kv_heads).
 *   out = softmax(scale q k^T) v,  lse = log sum e^{scale q k^T}
 *   q, k, v     device, bf16 or f16; token t, head h at element offset t*token_stride + h*head_stride,
 *               head_dim values in a row (slices of one fused projection output are fine).  Bases on
 *               16-byte boundaries, strides multiples of 8 and above 0
 *   head_dim    a multiple of 8, at most DISC_MAX_HEAD_DIM
 *   n_q_heads   a multiple of n_kv_heads, at most 128 times as many
 *   n_q, n_k    tokens in q and in k / v
 *   cu_q        device, int32[n_seqs+1], ascending from 0 to n_q;  cu_k the same over n_k (nullable:
 *               the same sequences)
 *   max_q       no sequence has more queries than this (sizes the launch)
 *   out         device, [n_q][n_q_heads][head_dim] contiguous, 16-byte aligned
 *   lse_out     device, float[n_q][n_q_heads] (nullable)
 *   error       device, 4 bytes: set to 1 when a bounded wait inside the kernel ran out (results
 *               invalid), never cleared; read with disc_attend_error
 * Scores, sums and outputs are accumulated in fp32; the probabilities are rounded to the inputs' type for
 * the second product, the outputs once at the end.  Non-finite keys and values do not reach queries that do not see
 * them, of the same sequence or another (but for an output that a value it sees makes infinite: it may come out as NaN).
 * Errors: DISC_ERR_ARG, DISC_ERR_UNSUPPORTED (dtype, head_dim, strides, head counts). */
#define DISC_MAX_HEAD_DIM 128
int disc_attend_prompt(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                       int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride, disc_dtype_t dtype,
                       int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_q, int64_t n_k, const int32_t* cu_q,
                       const int32_t* cu_k, int32_t n_seqs, int32_t max_q, int32_t causal, float scale, void* out, float* lse_out,
                       uint32_t* error, void* stream);

/* Synchronises `stream`; DISC_ERR_CUDA when an attention kernel has set this error word. */
int disc_attend_error(const uint32_t* error, void* stream);

/* ---- head norms and rotation of queries and keys ---------------------------------------------------
 * For every vector x of D = head_dim values, w = q_weight or k_weight:
 *   u = w x / sqrt(mean(x^2) + eps) with `norm` (a null weight counts as 1), u = x without
 *   y_a = u_a cos t_i - u_b sin t_i,  y_b = u_b cos t_i + u_a sin t_i,   t_i = position * inv_freq[i],  i < rot / 2
 * with (a, b) = (i, i + rot/2), or (2i, 2i + 1) with `interleaved`; values from rot on are not rotated.  Rounded once, at the end.
 * Angles are formed less their whole turns, in whole numbers: as exact at position 10^6 as at 10; a pair whose frequency is not finite
 * becomes NaN.  Sums of squares are held in fp32: |x| up to about 10^18, and with eps = 0 from about 10^-18.
 *
 * The call's arguments, in host memory, read before the call returns; what a call does not mention is not looked at. */
typedef struct {
    const void *q, *k, *v;     /* device, [n_tokens][heads][head_dim]: token t, head h at element offset t*token + h*head;           */
    void *q_out, *k_out;       /* bases on 16-byte boundaries, strides multiples of 8 (over an axis of one: any)                     */
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, q_out_token, q_out_head, k_out_token, k_out_head;
    const int32_t* positions;  /* device, int32[n_tokens]                                                                            */
    const float* inv_freq;     /* device, float[rot / 2] (nullable with rot = 0)                                                     */
    const void *q_weight, *k_weight;   /* device, head_dim values (nullable), 16-byte aligned                                        */
    int64_t n_tokens;
    const int32_t *cu, *rows;  /* disc_norm_rope_write: as for disc_cache_write                                                      */
    const uint8_t* status;
    int32_t dtype;             /* DISC_BF16 or DISC_F16                                                                              */
    int32_t n_q_heads, n_kv_heads;     /* 0: without queries, without keys                                                           */
    int32_t head_dim;          /* a multiple of 8, at most DISC_MAX_HEAD_DIM                                                         */
    int32_t rot;               /* a multiple of 8, at most head_dim; 0: no rotation                                                  */
    int32_t interleaved, norm; /* 0 or 1                                                                                             */
    int32_t weight_dtype;      /* DISC_F32 or the vectors' type                                                                      */
    float eps;                 /* >= 0                                                                                               */
    int32_t n_seqs;
} disc_norm_rope_t;

/* q -> q_out, k -> k_out, by the tokens' positions (nullable with rot = 0).  An output may be its own input (same strides); otherwise it
 * must not overlap any input, nor the other output.
 * Errors: DISC_ERR_ARG (also for an output that begins where another input does), DISC_ERR_UNSUPPORTED (dtype, head_dim, rot, strides, weight_dtype). */
int disc_norm_rope(const disc_norm_rope_t* a, void* stream);

/* Its gradient: q_out, k_out are the gradients of the results (read; strides of 0 allowed), from which come those of q and k
 * and, where not null, of the weights.
 *   d_q, d_k    device, [n_tokens][heads][head_dim] contiguous, 16-byte aligned, of the vectors' type; must not overlap any input
 *   d_q_weight, d_k_weight   device, float[head_dim] (nullable; need `norm`): sums in fp32, the same every time
 *   scratch     device, disc_norm_rope_scratch_bytes() bytes, 4-byte aligned (nullable without weight gradients) */
int64_t disc_norm_rope_scratch_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_tokens);
int disc_norm_rope_grad(const disc_norm_rope_t* a, void* d_q, void* d_k, float* d_q_weight, float* d_k_weight, void* scratch,
                        int64_t scratch_bytes, void* stream);

/* ---- the key-value cache ---------------------------------------------------------------------------
 * Rows (sequences) hold their keys and values in pages of page_size tokens; a page may belong to several
 * rows, which is how the K candidates of a query share its prompt.  All memory is the caller's, on
 * the device; the struct itself is host memory and may be rebuilt for every call.
 *   pool    [n_layers][2][n_pages][n_kv_heads][page_size][head_dim] of dtype (index 1: keys, values)
 *   table   int32[n_rows][table_width]: the pages of row r in order; -1 beyond the last one
 *   len     int32[n_rows]: tokens of row r; it uses ceil(len / page_size) pages
 *   ref     int32[n_pages]: number of table entries that name the page; 0 = free
 *   scratch disc_cache_scratch_bytes() bytes, 16-byte aligned, contents irrelevant between calls
 * An empty cache has table = -1, len = 0, ref = 0.  The calls below keep the three consistent; new
 * pages are always the free ones of lowest id.  The calls on one cache must not overlap on the device.
 * Page sizes: 16, 32, 64, 128.  dtype bf16 or f16, head_dim a multiple of 8 up to 128.
 *
 * With dtype | DISC_HELD_E4M3 or | DISC_HELD_I8 the vectors, of type bf16 or f16 where they are given and returned, are held in 8
 * bits: one code per value and a power of two, 2^e, per vector.  head_dim is then a multiple of 16 and
 *   pool    [n_layers][2][n_pages][n_kv_heads] parts of page_size * (head_dim + 1) bytes: the codes [page_size][head_dim], then
 *           the exponents, one signed byte per token
 *   e4m3    e = floor(log2 amax) - 8, one more where amax 2^-e > 448;  amax: the vector's largest |value|
 *   i8      e = floor(log2 amax) - 6, one more where amax 2^-e rounds to more than 127;  two's complement
 *   code    value * 2^-e rounded to the nearest, ties to even;  e is at least -126
 * so that an e4m3 code is off by at most 2^-4 of its value (or 2^-10 2^e), an i8 code by half of 2^e.  A held value, code * 2^e, is exact in the
 * vectors' type; one that exceeds the type's largest finite value (an e4m3 code rounded up) is given back as that.  A vector
 * with an infinite value or a NaN is held as e = -128 and reads as NaN throughout.  In a pool that is filled otherwise, e4m3 codes of
 * 0x7f and 0xff, which are no numbers, have no place. */
#define DISC_HELD_E4M3 0x10
#define DISC_HELD_I8 0x20
typedef struct {
    void* pool;
    int32_t* table;
    int32_t* len;
    int32_t* ref;
    void* scratch;
    int64_t scratch_bytes;
    int32_t n_layers, n_pages, n_kv_heads, page_size, head_dim, n_rows, table_width, dtype;
} disc_cache_t;

int64_t disc_cache_scratch_bytes(const disc_cache_t* c);   /* from the sizes alone */

/* Row r becomes what row parent[r] was before the call, sharing its pages (no contents are copied); a
 * parent outside [0, n_rows) empties the row.  Any mapping is allowed: fork K candidates from
 * a prompt, reorder, keep the drawn candidate of each query and drop the others.
 *   parent  device, int32[n_rows]; parent[r] = r leaves the row as it is */
int disc_cache_fork(const disc_cache_t* c, const int32_t* parent, void* stream);

/* The rows with freed[r] != 0 become empty.  freed: device, uint8[n_rows]. */
int disc_cache_free(const disc_cache_t* c, const uint8_t* freed, void* stream);

/* Room for add[r] more tokens in row r (add: device, int32[n_rows]; null = one each; <= 0 = none): len
 * grows, new pages are taken, and a row about to write into a partly filled page that other rows hold too
 * gets its own copy of the tokens in it, in all layers (when every holder of the page writes on, the longest of
 * them, of equally long ones the lowest row, keeps it).  Rows are served in ascending order: once the pages still
 * needed by a row and those before it exceed the free ones, that row and later ones that need a page get DISC_ROW_NOPAGE and stay as they
 * are; so do rows that would outgrow the table.  status_out: device, uint8[n_rows]. */
int disc_cache_extend(const disc_cache_t* c, const int32_t* add, uint8_t* status_out, void* stream);

/* Keys and values of the newest tokens of some rows into layer `layer`: sequence i of n_seqs is row rows[i]
 * (null: row i), its tokens t = cu[i] .. cu[i+1]-1 (null cu: one token, t = i) are the last ones
 * the row was extended by.
 *   k, v    device, token t, head h at element offset t*token_stride + h*head_stride; bases on
 *           16-byte boundaries, strides multiples of 8
 *   status  device, uint8[n_rows] (nullable): rows with a status (disc_cache_extend) are skipped
 * Into 8 bits: DISC_ERR_UNSUPPORTED for more than 2048 key heads. */
int disc_cache_write(const disc_cache_t* c, int32_t layer, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                     int64_t v_token_stride, int64_t v_head_stride, int64_t n_tokens, const int32_t* cu, int32_t n_seqs,
                     const int32_t* rows, const uint8_t* status, void* stream);

/* Tokens of some rows out of layer `layer`, packed: token t = cu[i] + j of sequence i (row rows[i]; null: row i) is token
 * start[i] + j (null start: j) of its row; places before cu[0] and from cu[n_seqs] on are left as they are.
 *   cu       device, int32[n_seqs+1], ascending, cu[n_seqs] <= n_tokens
 *   k_out, v_out   device, [n_tokens][n_kv_heads][head_dim] contiguous, 32-byte aligned; zeros for tokens the row does not have
 * Errors: DISC_ERR_ARG, DISC_ERR_UNSUPPORTED (also for tokens of more than 2^15 runs of 16 bytes). */
int disc_cache_read(const disc_cache_t* c, int32_t layer, const int32_t* cu, int32_t n_seqs, const int32_t* rows, const int32_t* start, int64_t n_tokens,
                    void* k_out, void* v_out, void* stream);

/* disc_norm_rope on the newest tokens' queries and keys (n_kv_heads, head_dim and dtype are the cache's), and disc_cache_write of the
 * resulting keys and of v as they are, in one launch and bit for bit what the two give.
 *   positions   nullable: each token's place in its row, 0 for one that has none
 *   k_out       not used
 * cu, n_seqs, rows, status as for disc_cache_write; the queries of tokens that are not written are formed all the same. */
int disc_norm_rope_write(const disc_cache_t* c, int32_t layer, const disc_norm_rope_t* a, void* stream);

/* The n pages in use move to the ids 0 .. n-1 (those that are there already stay, the others go to
 * the free ids below n in order), contents of all layers with them.  live_out: device, int32: n. */
int disc_cache_compact(const disc_cache_t* c, int32_t* live_out, void* stream);

/* ---- attention of one new token per row over the cache -----------------------------------------------
 * The plan: which pages each group of `group` consecutive rows (K candidates of a query; 1 = unrelated
 * rows) has in common, and how the work is split.  It depends on the books only: make it once per position, after
 * disc_cache_extend, and use it for every layer.
 *   plan    device, disc_attend_plan_bytes() bytes, 32-byte aligned.  Its first 4 bytes are an error word as
 *           disc_attend_prompt's: the caller sets it to 0 before the first plan is made in the buffer, disc_attend_cached sets
 *           it to 1, and no call clears it, so that it can be read (disc_attend_error) once after many positions
 * Errors: DISC_ERR_ARG; DISC_ERR_UNSUPPORTED for more than 64 query heads per key head, or tables of more than 2^30 blocks of
 * 16 tokens. */
int64_t disc_attend_plan_bytes(const disc_cache_t* c, int32_t n_q_heads, int32_t group);
int disc_attend_plan(const disc_cache_t* c, int32_t n_q_heads, int32_t group, void* plan, int64_t plan_bytes, void* stream);

/* out[r] = softmax(scale q[r] K^T) V over the len[r] tokens of row r in layer `layer`; a row without tokens
 * gets out = 0, lse = -inf.  Pages that the rows with tokens of a group have in common are read once for all of them (for groups
 * of more than 128 query vectors, rows times the query heads of a key head, once for each 128 or so).
 *   q       device, dtype of the cache; row r, head h at element offset r*q_row_stride + h*q_head_stride;
 *           base on a 16-byte boundary, strides multiples of 8 and above 0 (up to 16 query vectors per group, min(group, n_rows) times
 *           the query heads of a key head, any multiples)
 *   n_q_heads   a multiple of n_kv_heads, at most 64 times as many
 *   scale   > 0
 *   plan    of disc_attend_plan with the same cache sizes, n_q_heads and group; long rows are split and joined in
 *           it, so calls that share a plan must not overlap
 *   out     device, [n_rows][n_q_heads][head_dim] contiguous, 16-byte aligned
 *   lse_out device, float[n_rows][n_q_heads] (nullable)
 * Scores, sums and outputs are accumulated in fp32; the probabilities are rounded to the inputs' type (f16: with steps of 2^-24 of the
 * largest at their lower end) for the second product (up to 8 query vectors per group, min(group, n_rows) times the query heads of a key head: to twice its
 * digits), the outputs once at the end.  The result does not depend on the order in which the parts of
 * a row finish, and a row's non-finite values do not reach the other rows of its group.
 * Over a cache held in 8 bits the values that are held take part as they are; outputs beyond f16's largest value are given as that.  Up to
 * 16 query vectors per group the probabilities, times the values' powers of two, are rounded to f16 relative to 2^7 times the largest of
 * them (what is below 2^-32 of that one is lost; q of type f16: to twice its digits), above that as over 16 bits;
 * a vector held as NaN makes NaN of all outputs of the query heads that see it. */
int disc_attend_cached(const disc_cache_t* c, int32_t layer, const void* q, int64_t q_row_stride, int64_t q_head_stride,
                       int32_t n_q_heads, int32_t group, float scale, void* plan, int64_t plan_bytes, void* out, float* lse_out,
                       void* stream);

/* Diagnostic: the n group-noise uniforms of token groups g0 .. g0+n-1 for (seed, step, row), fp32.
 *   out  device, float[n] */
int disc_sampling_uniforms(uint64_t seed, uint32_t step, uint32_t row, int32_t g0, int32_t n,
                           float* out, void* stream);

/* Text for a DISC_ERR_* code. */
const char* disc_error_string(int code);

/* cudaError_t (as int) of the most recent failed CUDA call made by this library on this thread. */
int disc_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DISC_H_ */
